// Cross-entropy of a linear head, and its gradients, without the logits in
// memory (atom_k_linear_xent_fwd, atom_k_linear_xent_bwd).
//
//   z = x W^T,  lse_n = log sum_v exp z_nv,  loss_n = lse_n - z_n[t_n]
//   dz_nv = (exp(z_nv - lse_n) - [v = t_n]) drow_n,  dx = scale dz W,
//   dW = scale dz^T x
//
// Forward: one product whose epilogue (EPI_LSE, gemm_dl.h) turns the logits of
// a wave's block, still in the accumulators, into a maximum and a sum of
// exponentials per row, and keeps the logit at the row's target; a second
// kernel joins a row's parts in their order.  Memory: x and W read, 8 bytes per
// token and part written and read.
// Backward: pieces of the vocabulary.  Per piece the logits are computed again,
// become dz in the epilogue (EPI_DZ) and go to the workspace in the element
// type, and two products read them: dx gains dz W (fp32 between pieces), and the
// piece's rows of dW = dz^T x are done.  A piece of dz that fits the 256 MB
// Infinity Cache is read from there.
//
// dz is held without `scale`, which multiplies the fp32 sums: the usual scale
// 1 / tokens is no power of two, and rounding -scale at the target would put a
// bf16 rounding error into every row's largest term, where -1 + p with a small
// p has next to none (2.4e-3 -> 1.7e-3 relative, the rounding of the result).
#include <algorithm>

#include "common.h"
#include "launch.h"

namespace atom {
namespace {

constexpr float LOG2E = 1.4426950408889634f;

// RPB rows per workgroup, 256 / RPB threads per row, each over every
// (256 / RPB)-th part; the threads' (max, sum) pairs join in LDS in a fixed
// order.  16 rows read 128 bytes of a part's row; few rows take a workgroup each.
// (A loop over the rows: 2^28 of them are more workgroups than a dispatch counts.)
template <int RPB>
__global__ void __launch_bounds__(256) lse_join_kernel(const float2* __restrict__ part, int64_t rows, int parts,
                                                       const int32_t* __restrict__ tgt,
                                                       const float* __restrict__ ztgt, int V,
                                                       float* __restrict__ lse, float* __restrict__ loss_rows) {
  constexpr int TPR = 256 / RPB;
  __shared__ float2 red[TPR][RPB];
  const int r = threadIdx.x % RPB, s = threadIdx.x / RPB;
  for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * RPB; row0 < rows; row0 += static_cast<int64_t>(gridDim.x) * RPB) {
    const int64_t row = row0 + r;
    float m = -INFINITY, sum = 0.f;
    if (row < rows) {
#pragma unroll 4
      for (int p = s; p < parts; p += TPR) {
        const float2 v = part[static_cast<int64_t>(p) * rows + row];
        const float n = fmaxf(m, v.x);
        const float ref = n == -INFINITY ? 0.f : n;
        sum = sum * __builtin_amdgcn_exp2f((m - ref) * LOG2E) + v.y * __builtin_amdgcn_exp2f((v.x - ref) * LOG2E);
        m = n;
      }
    }
    red[s][r] = make_float2(m, sum);
    __syncthreads();
#pragma unroll
    for (int h = TPR / 2; h > 0; h >>= 1) {
      if (s < h) {
        const float2 a = red[s][r], b = red[s + h][r];
        const float n = fmaxf(a.x, b.x);
        const float ref = n == -INFINITY ? 0.f : n;
        red[s][r] = make_float2(n, a.y * __builtin_amdgcn_exp2f((a.x - ref) * LOG2E) +
                                       b.y * __builtin_amdgcn_exp2f((b.x - ref) * LOG2E));
      }
      __syncthreads();
    }
    if (s == 0 && row < rows) {
      const int t = tgt[row];
      float l = 0.f, loss = 0.f;
      if (t >= 0) {
        const float m = red[0][r].x, g = logf(red[0][r].y);
        l = m + g;
        // not l - z: what l rounds off would be all of the loss of a token whose
        // target has nearly the whole sum
        loss = t < V ? (m - ztgt[row]) + g : NAN;
      }
      lse[row] = l;
      loss_rows[row] = loss;
    }
    __syncthreads();  // red
  }
}

// x with the rows of tokens that take no part set to zero, so that whatever
// they hold stays out of dz (their logits are zero) and of dW (dz is zero there,
// and 0 * NaN is not).
__global__ void __launch_bounds__(256) keep_rows_kernel(const uint4* __restrict__ x, int64_t ldc, int cpr,
                                                        const int32_t* __restrict__ tgt,
                                                        const float* __restrict__ drow, int64_t n,
                                                        uint4* __restrict__ y) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = i / cpr;
    const bool on = tgt[row] >= 0 && !(drow && drow[row] == 0.f);
    y[i] = on ? x[row * ldc + (i - row * cpr)] : make_uint4(0, 0, 0, 0);
  }
}

// Rows of an fp32 matrix as three bf16 planes [rows][dp], zeros from column d
// on; with tgt, rows that take no part are zero, as above.
__global__ void __launch_bounds__(256) planes_kernel(const float* __restrict__ x, int64_t ldx, int d, int dp,
                                                     const int32_t* __restrict__ tgt, const float* __restrict__ drow,
                                                     int64_t n, bf16_t* __restrict__ y, int64_t plane) {
  const int cpr = dp / 8;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = i / cpr;
    const int c = static_cast<int>(i - row * cpr) * 8;
    const bool on = !tgt || (tgt[row] >= 0 && !(drow && drow[row] == 0.f));
    uint2 p[2][3];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // d is a multiple of 4
      const float4 v = on && c + 4 * h < d ? *reinterpret_cast<const float4*>(x + row * ldx + c + 4 * h) : make_float4(0.f, 0.f, 0.f, 0.f);
      const float f[4] = {v.x, v.y, v.z, v.w};
      pack_three(f, p[h]);
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
      *reinterpret_cast<uint4*>(y + k * plane + row * dp + c) = make_uint4(p[0][k].x, p[0][k].y, p[1][k].x, p[1][k].y);
  }
}

__global__ void __launch_bounds__(256) zero_rows_kernel(uint32_t* __restrict__ y, int64_t ldw, int wpr, int64_t n) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256)
    y[i / wpr * ldw + i % wpr] = 0;
}

inline uint64_t up(uint64_t n) { return (n + 255) & ~255ull; }
inline unsigned blocks(int64_t n) { return static_cast<unsigned>(std::min<int64_t>((n + 255) / 256, 4096)); }
inline int esize(int dtype) { return dtype == DT_BF16 ? 2 : 4; }

// Whether fp32 operands become three bf16 planes (x = h + m + l, 24 bits), with
// six passes of bf16 MFMAs at two to three times the rate of fp32 ones: w's
// planes, 16 bytes of memory traffic an entry, want rows and work to pay for
// them.  54 problems, fp32 MFMAs against planes: loss 4096 x 512, vocabulary
// 8000, 309 and 190 us; 1024 x 512, 8000, 85 and 75; 512 x 512, 8000, 47 and 55; 1024 x
// 2048, 1000, 45 and 87; gradients 4096 x 2048, 8000, 3336 and 2087; 512 x 2048,
// 8000, 460 and 358; 256 x 2048, 50257, 1461 and 1737; 1024 x 128, 50257, 455 and 619.
bool planes(int dtype, int64_t rows, int V, int d, bool grad) {
  return dtype == DT_F32 && rows >= (grad ? 512 : 768) && d >= (grad ? 256 : 1) &&
         static_cast<double>(rows) * V * d >= 4294967296.0;
}
// Columns of a row of planes, an odd number of 128-byte lines.
int plane_ld(int d) { return ((d + 63) / 64 | 1) * 64; }
// Rows of w that are planes at a time (forward): equal parts of 192 MB at most,
// 1024 rows at least.
int plane_rows(int V, int d) {
  const int64_t most = std::max<int64_t>(1024, (192ll << 20) / (6 * plane_ld(d)) / 256 * 256), n = (V + most - 1) / most;
  return static_cast<int>(std::min<int64_t>(V, ((V + n - 1) / n + 255) / 256 * 256));
}
GemmArgs plane_args(const bf16_t* A, int64_t lda, int64_t pa, const bf16_t* B, int64_t ldb, int64_t pb, int M, int N, int K) {
  GemmArgs g{};
  g.A = A, g.lda = lda, g.B = B, g.ldb = ldb;
  g.M = M, g.N = N;
  g.pl = PlaneArgs{pa, pb, 0, (K + 31) / 32, K};
  g.K = 6 * 32 * g.pl.kp;
  return g;
}
hipError_t to_planes(const void* x, int64_t ldx, int64_t rows, int d, const int32_t* tgt, const float* drow, bf16_t* y,
                     hipStream_t s) {
  const int dp = plane_ld(d);
  const int64_t n = rows * (dp / 8);
  hipLaunchKernelGGL(planes_kernel, dim3(blocks(n)), dim3(256), 0, s, static_cast<const float*>(x), ldx, d, dp, tgt,
                     drow, n, y, rows * dp);
  return hipGetLastError();
}

// The pieces of the vocabulary: `width` columns each, the last one what is left.
struct Pieces {
  int width, last;  // last: columns of the last piece, at most 9/8 width
  int next(int v0, int V) const { return V - v0 <= last ? V - v0 : width; }
};

// The caller's width, or by default the whole vocabulary where dz of it takes
// at most 128 MB, half of the Infinity Cache, through which the two products
// read it, else the largest power of two from 2048 to 16384 within that.  A
// narrow d reads dz less often, and short pieces cost it more: 256 MB, and 512
// for the piece.  Vocabulary 50257, pieces of 4096, 8192, 16384, 32768: 2048 x
// 5120 3306, 2784, 2658, 2815 us; 4096 x 4096 4129, 3955, 3971, 3958; 999 x 2048
// 1039, 787, 679, 636, whole 600; 16384 x 768 3849, 3711, 3589, 3553.  Within
// 128 MB and as here: 1500 x 2048 1003 and 942; 32768 x 768 8212 and 7179; 16384 x
// 2560 11143 and 10491; but whole, 4096 x 2560 (412 MB) 2720 and 2822, 2048 x 5120
// (206 MB) 2659 and 2786.  A short rest joins the last piece.  (Three planes:
// bytes of dz or of w's planes; 600 x 2048 2923 and 2595.)
Pieces pieces_of(int dtype, int64_t rows, int V, int d, int piece) {
  if (piece > 0) {
    const int w = static_cast<int>(std::min<int64_t>(V, (piece + 7ll) / 8 * 8));
    return Pieces{w, w};
  }
  const bool narrow = d <= 2560;
  const int64_t column = planes(dtype, rows, V, d, true) ? 6 * std::max<int64_t>(rows, plane_ld(d)) : rows * esize(dtype);
  if (V <= (narrow ? 256ll << 20 : 128ll << 20) / column) return Pieces{V, V};
  int w = 16384;
  while (w > 2048 && w > (narrow ? 512ll << 20 : 128ll << 20) / column) w /= 2;
  w = std::min(V, w);
  const int rest = V % w;
  return Pieces{w, rest > 0 && rest <= w / 8 ? w + rest : w};
}

// Workspace for few rows: ranges of the vocabulary summed apart (dx), up to 16
// in 64 MB (32, 64, 128 MB: 999 x 4096, vocabulary 50257, 1280, 1212, 1178 us; 1500 x
// 2048 1030, 988, 982; 512 x 4096 741, 699, 697; 2048 x 5120 2735, 2745, 2797).
uint64_t split_bytes(int64_t rows, int d) { return std::min<uint64_t>(up(16ull * rows * d * 4), 64ull << 20); }

// Rows of dz start an odd number of 256-byte lines apart: pieces are multiples
// of 4 KB or more, and rows that far apart crowd a few memory channels.
int ld_of_dz(int esz, int piece) {
  const int line = 256 / esz;
  return ((piece + line - 1) / line | 1) * line;
}

struct BwdWs {
  uint64_t dz, x, w, dx, split, split_bytes, end;  // offsets
};
BwdWs bwd_ws(int dtype, int64_t rows, int V, int d, const Pieces& p) {
  const bool three = planes(dtype, rows, V, d, true);
  const uint64_t e = three ? 6 : esize(dtype), n = rows;
  const int ldz = ld_of_dz(three ? 2 : esize(dtype), p.last);
  const uint64_t wide = three ? plane_ld(d) : d;
  BwdWs w;
  w.dz = 0;
  w.x = w.dz + up(n * ldz * e);
  w.w = w.x + up(n * wide * e);
  w.dx = w.w + (three ? up(p.last * wide * e) : 0);
  w.split = w.dx + (dtype == DT_BF16 && p.last < V ? up(n * d * 4) : 0);
  w.split_bytes = split_bytes(rows, d);
  w.end = w.split + w.split_bytes;
  return w;
}

}  // namespace

// Lengths whose tiles (32 x 32 at least) and passes over k are counted in 32 bits.
bool linear_xent_ok(int dtype, int64_t rows, int V, int d) {
  if (rows < 0 || rows > (1 << 28) || V <= 0 || V > (1 << 28) || d <= 0 || d > (1 << 24)) return false;
  if (d % (dtype == DT_BF16 ? 8 : 4)) return false;
  const int64_t tr = (rows + 31) / 32, tv = (static_cast<int64_t>(V) + 31) / 32, td = (d + 31) / 32;
  return tr * tv < (1ll << 30) && tv * td < (1ll << 30) && tr * td < (1ll << 30);
}

namespace {
struct FwdWs {
  uint64_t ztgt, x, w, part, end;  // offsets
  int64_t parts;
  int range;  // rows of w at a time
};
FwdWs fwd_ws(int dtype, int64_t rows, int V, int d) {
  FwdWs w;
  const bool three = planes(dtype, rows, V, d, false);
  const int m = static_cast<int>(rows);
  w.range = three ? plane_rows(V, d) : V;
  w.parts = 0;
  for (int v0 = 0; v0 < V; v0 += w.range) {
    const int n = std::min(w.range, V - v0);
    w.parts += three ? gemm_lse_parts(DT_BF16, m, n, 6 * 32 * ((d + 31) / 32)) : gemm_lse_parts(dtype, m, n, d);
  }
  w.ztgt = 0;
  w.x = up(rows * sizeof(float));
  w.w = w.x + (three ? up(6ull * rows * plane_ld(d)) : 0);
  w.part = w.w + (three ? up(6ull * w.range * plane_ld(d)) : 0);
  w.end = w.part + w.parts * rows * sizeof(float2);
  return w;
}
}  // namespace

bool linear_xent_fwd_ok(int dtype, int64_t rows, int V, int d) {
  if (!linear_xent_ok(dtype, rows, V, d)) return false;
  if (rows == 0) return true;
  const int m = static_cast<int>(rows);
  if (!planes(dtype, rows, V, d, false)) return gemm_lse_fits(dtype, m, V, d);
  const int range = plane_rows(V, d), k = 6 * 32 * ((d + 31) / 32), rest = V % range;
  return gemm_lse_fits(DT_BF16, m, range, k) && (rest == 0 || gemm_lse_fits(DT_BF16, m, rest, k));
}

uint64_t linear_xent_fwd_ws(int dtype, int64_t rows, int V, int d) {
  return rows == 0 ? 0 : fwd_ws(dtype, rows, V, d).end;
}

hipError_t linear_xent_fwd(int dtype, const void* x, int64_t ldx, const void* w, int64_t ldw, const int32_t* tgt,
                           float* lse, float* loss_rows, int64_t rows, int V, int d, void* ws, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const FwdWs o = fwd_ws(dtype, rows, V, d);
  char* base = static_cast<char*>(ws);
  float* ztgt = reinterpret_cast<float*>(base + o.ztgt);
  float2* part = reinterpret_cast<float2*>(base + o.part);
  const int m = static_cast<int>(rows);
  hipError_t e;
  if (planes(dtype, rows, V, d, false)) {
    const int dp = plane_ld(d);
    bf16_t *xp = reinterpret_cast<bf16_t*>(base + o.x), *wp = reinterpret_cast<bf16_t*>(base + o.w);
    e = to_planes(x, ldx, rows, d, nullptr, nullptr, xp, s);
    float2* at = part;
    for (int v0 = 0; v0 < V && e == hipSuccess; v0 += o.range) {
      const int n = std::min(o.range, V - v0);
      e = to_planes(static_cast<const float*>(w) + v0 * ldw, ldw, n, d, nullptr, nullptr, wp, s);
      if (e != hipSuccess) return e;
      GemmArgs g = plane_args(xp, dp, rows * dp, wp, dp, static_cast<int64_t>(n) * dp, m, n, d);
      g.ztgt = ztgt, g.C = at, g.tgt = tgt, g.v0 = v0, g.V = V;
      e = gemm_loss(g, dtype, true, true, EPI_LSE, s);
      at += gemm_lse_parts(DT_BF16, m, n, g.K) * rows;
    }
  } else {
    GemmArgs g{};
    g.A = x, g.lda = ldx, g.B = w, g.ldb = ldw;
    g.M = m, g.N = V, g.K = d;
    g.ztgt = ztgt, g.C = part, g.tgt = tgt, g.V = V;
    e = gemm_loss(g, dtype, true, true, EPI_LSE, s);
  }
  if (e != hipSuccess) return e;
  if (rows < 2048)
    hipLaunchKernelGGL(lse_join_kernel<1>, dim3(static_cast<unsigned>(rows)), dim3(256), 0, s, part, rows,
                       static_cast<int>(o.parts), tgt, ztgt, V, lse, loss_rows);
  else
    hipLaunchKernelGGL(lse_join_kernel<16>, dim3(static_cast<unsigned>(std::min<int64_t>((rows + 15) / 16, 1 << 20))),
                       dim3(256), 0, s, part, rows, static_cast<int>(o.parts), tgt, ztgt, V, lse, loss_rows);
  return hipGetLastError();
}

uint64_t linear_xent_bwd_ws(int dtype, int64_t rows, int V, int d, int piece) {
  return rows == 0 ? 0 : bwd_ws(dtype, rows, V, d, pieces_of(dtype, rows, V, d, piece)).end;
}

hipError_t linear_xent_bwd(int dtype, const void* x, int64_t ldx, const void* w, int64_t ldw, const int32_t* tgt,
                           const float* lse, const float* drow, float scale, void* dx, int64_t lddx, void* dw,
                           int64_t lddw, int dw_epi, int64_t rows, int V, int d, int piece, void* ws, hipStream_t s) {
  const int esz = esize(dtype);
  const int wsz = dw_epi == EPI_SCALE ? esz : 4;  // bytes of an element of dw
  if (rows == 0) {
    if (!dw || dw_epi == EPI_SCALE_ACC) return hipSuccess;
    const int wpr = d * wsz / 4;
    const int64_t n = static_cast<int64_t>(V) * wpr;
    hipLaunchKernelGGL(zero_rows_kernel, dim3(blocks(n)), dim3(256), 0, s, static_cast<uint32_t*>(dw), lddw * wsz / 4,
                       wpr, n);
    return hipGetLastError();
  }
  const Pieces pc = pieces_of(dtype, rows, V, d, piece);
  const BwdWs o = bwd_ws(dtype, rows, V, d, pc);
  char* base = static_cast<char*>(ws);
  const bool three = planes(dtype, rows, V, d, true);
  const int ldz = ld_of_dz(three ? 2 : esize(dtype), pc.last);
  char* xz = base + o.x;
  if (three) {
    const int dp = plane_ld(d), m = static_cast<int>(rows);
    bf16_t *zp = reinterpret_cast<bf16_t*>(base), *xp = reinterpret_cast<bf16_t*>(xz), *wp = reinterpret_cast<bf16_t*>(base + o.w);
    const int64_t px = rows * dp, pz = rows * ldz;
    hipError_t e = to_planes(x, ldx, rows, d, tgt, drow, xp, s);
    for (int v0 = 0, n; v0 < V && e == hipSuccess; v0 += n) {
      n = pc.next(v0, V);
      const int64_t pw = static_cast<int64_t>(n) * dp;
      e = to_planes(static_cast<const float*>(w) + v0 * ldw, ldw, n, d, nullptr, nullptr, wp, s);
      if (e != hipSuccess) return e;
      GemmArgs g = plane_args(xp, dp, px, wp, dp, pw, m, n, d);
      g.C = zp, g.ldc = ldz, g.pl.pc = pz;
      g.tgt = tgt, g.lse = lse, g.rowscale = drow, g.v0 = v0, g.V = V;
      e = gemm_loss(g, dtype, true, true, EPI_DZ, s);
      if (e == hipSuccess && dx) {
        GemmArgs a = plane_args(zp, ldz, pz, wp, dp, pw, m, d, n);
        a.C = dx, a.ldc = lddx, a.alpha = scale;
        a.ws = reinterpret_cast<float*>(base + o.split), a.ws_bytes = o.split_bytes;
        e = gemm_loss(a, dtype, true, false, v0 == 0 ? EPI_SCALE_F32 : EPI_SCALE_ACC, s);
      }
      if (e == hipSuccess && dw) {
        GemmArgs a = plane_args(zp, ldz, pz, xp, dp, px, n, d, m);
        a.C = static_cast<float*>(dw) + v0 * lddw, a.ldc = lddw, a.alpha = scale;
        a.ws = reinterpret_cast<float*>(base + o.split), a.ws_bytes = o.split_bytes;
        e = gemm_loss(a, dtype, false, false, dw_epi == EPI_SCALE_ACC ? EPI_SCALE_ACC : EPI_SCALE_F32, s);
      }
    }
    return e;
  }
  {
    const int cpr = d * esz / 16;
    const int64_t n = rows * cpr;
    hipLaunchKernelGGL(keep_rows_kernel, dim3(blocks(n)), dim3(256), 0, s, static_cast<const uint4*>(x),
                       ldx * esz / 16, cpr, tgt, drow, n, reinterpret_cast<uint4*>(xz));
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // the sum over the pieces: in dx itself (fp32), or beside it
  float* sum = dtype == DT_BF16 ? reinterpret_cast<float*>(base + o.dx) : static_cast<float*>(dx);
  const int64_t ldsum = dtype == DT_BF16 ? d : lddx;
  for (int v0 = 0, n; v0 < V; v0 += n) {
    n = pc.next(v0, V);
    const char* wp = static_cast<const char*>(w) + static_cast<int64_t>(v0) * ldw * esz;
    GemmArgs g{};
    g.A = xz, g.lda = d, g.B = wp, g.ldb = ldw, g.C = base, g.ldc = ldz;
    g.M = static_cast<int>(rows), g.N = n, g.K = d;
    g.tgt = tgt, g.lse = lse, g.rowscale = drow, g.v0 = v0, g.V = V;
    hipError_t e = gemm_loss(g, dtype, true, true, EPI_DZ, s);
    if (e != hipSuccess) return e;
    GemmArgs h{};
    h.A = base, h.lda = ldz;
    h.ws = reinterpret_cast<float*>(base + o.split), h.ws_bytes = o.split_bytes;
    h.N = d, h.alpha = scale;
    if (dx) {
      const bool first = v0 == 0, last = v0 + n == V;
      GemmArgs a = h;
      a.B = wp, a.ldb = ldw, a.M = static_cast<int>(rows), a.K = n;
      a.C = last ? dx : sum, a.ldc = last ? lddx : ldsum;
      a.resid = sum, a.ldaux = ldsum;
      if (!last) a.alpha = 1.f;
      e = gemm_loss(a, dtype, true, false, last ? (first ? EPI_SCALE : EPI_SUM_SCALE) : first ? EPI_STORE_F32 : EPI_SCALE_ACC, s);
      if (e != hipSuccess) return e;
    }
    if (dw) {
      GemmArgs a = h;
      a.B = xz, a.ldb = d, a.M = n, a.K = static_cast<int>(rows);
      a.C = static_cast<char*>(dw) + static_cast<int64_t>(v0) * lddw * wsz, a.ldc = lddw;
      e = gemm_loss(a, dtype, false, false, dw_epi, s);
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace atom

// What the sizes are worked on as (tests): whether in three planes, rows of w at
// a time (forward), columns of a piece and of the last one (backward), and the
// bytes for ranges of k (backward).
extern "C" void atom_linear_xent_plan(int dtype, int64_t rows, int V, int d, int piece, int64_t* out) {
  using namespace atom;
  out[0] = planes(dtype, rows, V, d, false), out[1] = out[0] ? plane_rows(V, d) : V;
  const Pieces p = pieces_of(dtype, rows, V, d, piece);
  out[2] = planes(dtype, rows, V, d, true), out[3] = p.width, out[4] = p.last;
  out[5] = static_cast<int64_t>(split_bytes(rows, d));
}
