// Newton-Schulz orthogonalisation of a matrix (atom_k_orthogonalize): the
// update of the Muon optimiser, U V^T of the singular value decomposition G =
// U S V^T but for the singular values, which end near 1 instead of at 1.
//
//   X = G / (|G|_F + 1e-7); per step  A = X X^T,  B = b A + c A^2,
//   X <- a X + B X;  with A = X^T X and X B for matrices taller than wide.
//
// Every step works on the singular values alone, s <- a s + b s^3 + c s^5.
// All products run on the direct-load kernel (gemm_dl.h) in fp16 MFMAs with
// fp32 sums, on matrices scaled by 2^10 (X also by a power of two per matrix
// and step, see pack_kernel) and padded with zeros to multiples of 32, and each
// step's sums and scalings are its products' epilogues: three launches a step,
// four where A is summed in ranges of k.  A and B are symmetric, so their
// products take the tiles on and below the diagonal.
//
// Precision.  X is kept as two fp16 planes, hi + lo (22 bits): rounding X to
// one would mix its strong directions into the weak ones, which later steps
// raise by up to a per step (a gradient of rank 8 over noise of 1e-3, 512 x
// 512: 4e-2 off in relative norm; 3e-4 with two planes).  The product B X may
// take hi alone where the result is bf16, because B is small where X's
// directions are weak, and so may A and B be one plane: the result is 1.7e-3 to
// 2.4e-3 from the definition, whose own rounding is 1.66e-3 off (fp16, with 11
// bits, not bf16: 1.5e-2).  fp32 results, of bf16 gradients too, take two planes
// of all three, and each product three passes over k (hi hi, hi lo, lo hi), at
// three eighths of the fp16 rate and still about three times that of fp32 MFMAs:
// 1.1e-6 to 4.7e-6 from the definition, fp32 arithmetic 1.7e-6 to 6.4e-6 (256 x
// 768 to 2048 x 8192 and 4096 x 4096; gradients of a few strong directions,
// Gaussian ones, singular values over four decades).
#include <algorithm>
#include <cmath>

#include "common.h"
#include "launch.h"

namespace atom {

hipError_t gemm_ns_256(const GemmArgs& g, int planes, int batch, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_ns_192(const GemmArgs& g, int planes, int batch, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_ns_128(const GemmArgs& g, int planes, int batch, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_ns_64(const GemmArgs& g, int planes, int batch, bool akc, bool bkc, int epi, hipStream_t s);

hipError_t gemm_ns(const GemmArgs& g, int bs, int planes, int batch, bool akc, bool bkc, int epi, hipStream_t s) {
  return bs == 256   ? gemm_ns_256(g, planes, batch, akc, bkc, epi, s)
         : bs == 192 ? gemm_ns_192(g, planes, batch, akc, bkc, epi, s)
         : bs == 128 ? gemm_ns_128(g, planes, batch, akc, bkc, epi, s)
                     : gemm_ns_64(g, planes, batch, akc, bkc, epi, s);
}

namespace {

constexpr float SCALE = 1024.f;  // of every fp16 matrix: entries of 2^-24 of the norm are still held
constexpr double EPS = 1e-7;
constexpr int NORM_BLOCKS = 1024;  // most partial sums of squares of a matrix

// Eight elements of a row from column c on, zeros from `cols` on.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int c, int cols, float* v) {
  if (VEC && c + 8 <= cols) {
    if constexpr (sizeof(T) == 2) {
      const uint4 w = *reinterpret_cast<const uint4*>(p + c);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) v[2 * k] = bf2f(u[k] & 0xffff), v[2 * k + 1] = bf2f(u[k] >> 16);
    } else {
      const float4 a = *reinterpret_cast<const float4*>(p + c), b = *reinterpret_cast<const float4*>(p + c + 4);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = c + k < cols ? to_f<T>(p[c + k]) : 0.f;
  }
}

// A workgroup takes 256 >> lx rows at a time, 1 << lx threads a row, eight
// columns a thread.  VEC: rows of g start on 16 bytes.
//
// Partial sums of squares in 64 bits: no entry's square over- or underflows,
// and long sums lose nothing.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) norm_kernel(const T* __restrict__ g, int64_t ldg, int64_t stride, int rows,
                                                   int cols, int lx, double* __restrict__ part) {
  __shared__ double red[4];
  g += blockIdx.y * stride;
  const int x = threadIdx.x & ((1 << lx) - 1), rpb = 256 >> lx;
  double s[2] = {0.0, 0.0};
  for (int r = blockIdx.x * rpb + (threadIdx.x >> lx); r < rows; r += gridDim.x * rpb) {
    const T* p = g + r * ldg;
#pragma unroll 4
    for (int c = 8 * x; c < cols; c += 8 << lx) {
      float v[8];
      load8<T, VEC>(p, c, cols, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k & 1] = fma(static_cast<double>(v[k]), static_cast<double>(v[k]), s[k & 1]);
    }
  }
  double t = s[0] + s[1];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.y * gridDim.x + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// Largest |a s + b s^3 + c s^5| of s in [0, top], from its extrema: a + 3 b x +
// 5 c x^2 = 0, x = s^2.  The root that -3 b and the discriminant's would cancel
// in is the product of the roots over the other one (c may be 0 or next to it).
__host__ __device__ inline double step_bound(double a, double b, double c, double top) {
  auto f = [=](double s) { return fabs(s * (a + s * s * (b + c * s * s))); };
  const double t = top * top, disc = 9 * b * b - 20 * a * c;
  double most = f(top);
  if (disc >= 0.0) {
    const double q = -0.5 * (3 * b + copysign(sqrt(disc), b)), x0 = q / (5 * c), x1 = a / q;
    if (x0 > 0.0 && x0 < t) most = fmax(most, f(sqrt(x0)));
    if (x1 > 0.0 && x1 < t) most = fmax(most, f(sqrt(x1)));
  }
  return most;
}

// The power of two that a matrix of norm at most r is held times: r 2^e in [1/2,
// 1); none for r of 1/2 and more, and 2^126 at most (a norm of 2^-150).
__host__ __device__ inline int exponent_of(double r) {
  if (!(r < 0.5 && r > 0.0)) return 0;
  const int e = -1 - ilogb(r);
  return e < 126 ? e : 126;
}

struct Steps {
  float coef[3 * NS_EXPS];
  int exps[NS_EXPS];  // of a norm of 1
  int n;
};

// X = SCALE * 2^e * g / (norm + EPS) in two planes [rp][cp], zeros past the
// matrix.  A norm that is not finite makes all of X NaN.  The EPS makes X small
// where the norm is far below it, and planes are fixed-point: 2^e, from the
// bound on the singular values, keeps their 22 bits.  exps: e of every step.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) pack_kernel(const T* __restrict__ g, int64_t ldg, int64_t stride, int rows,
                                                   int cols, int rp, int cp, int lx, const double* __restrict__ part,
                                                   int parts, Steps steps, int* __restrict__ exps,
                                                   f16_t* __restrict__ hi, f16_t* __restrict__ lo, int64_t sx) {
  __shared__ double red[4];
  g += blockIdx.y * stride;
  hi += blockIdx.y * sx;
  lo += blockIdx.y * sx;
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += 256) s += part[blockIdx.y * parts + i];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  s = (red[0] + red[1]) + (red[2] + red[3]);
  const double norm = sqrt(s), ratio = norm / (norm + EPS);
  const int e0 = exponent_of(ratio);
  const double f = s < INFINITY ? ldexp(SCALE / (norm + EPS), e0) : NAN;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    int* e = exps + blockIdx.y * NS_EXPS;
    e[0] = e0;
    double r = ratio;
    for (int k = 1; k < steps.n; ++k) {
      if (e0 > 0) r = step_bound(steps.coef[3 * k - 3], steps.coef[3 * k - 2], steps.coef[3 * k - 1], r);
      e[k] = e0 > 0 ? exponent_of(r) : steps.exps[k];
    }
  }
  const int x = threadIdx.x & ((1 << lx) - 1), rpb = 256 >> lx;
  for (int r = blockIdx.x * rpb + (threadIdx.x >> lx); r < rp; r += gridDim.x * rpb) {
    const T* p = g + r * ldg;
#pragma unroll 2
    for (int c = 8 * x; c < cp; c += 8 << lx) {
      float v[8];
      load8<T, VEC>(p, c, r < rows ? cols : 0, v);
      f16x8_t a, b;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float y = static_cast<float>(static_cast<double>(v[k]) * f);
        a[k] = static_cast<_Float16>(y);
        b[k] = static_cast<_Float16>(y - static_cast<float>(a[k]));
      }
      *reinterpret_cast<f16x8_t*>(hi + static_cast<int64_t>(r) * cp + c) = a;
      *reinterpret_cast<f16x8_t*>(lo + static_cast<int64_t>(r) * cp + c) = b;
    }
  }
}

// Threads a row (their logarithm) of the two kernels above, and partial sums of a
// matrix: a few thousand workgroups over the batch, since each workgroup of the
// second kernel sums all parts of its matrix.
int row_threads(int cols) {
  int lx = 0;
  while (lx < 8 && 8 << lx < cols) ++lx;
  return lx;
}
int norm_parts(int batch, int rows, int cols) {
  const int at_once = 256 >> row_threads(cols);  // rows of a workgroup
  return std::min(std::max(64, NORM_BLOCKS / batch), (rows + at_once - 1) / at_once);
}

template <typename T>
void launch_pack(const void* g, int64_t ldg, int64_t stride, int batch, int rows, int cols, int rp, int cp,
                 double* part, const Steps& steps, int* exps, f16_t* hi, f16_t* lo, hipStream_t s) {
  const T* p = static_cast<const T*>(g);
  const int e = 16 / static_cast<int>(sizeof(T));
  const bool vec = reinterpret_cast<uintptr_t>(g) % 16 == 0 && ldg % e == 0 && stride % e == 0;
  const int lx = row_threads(cols), parts = norm_parts(batch, rows, cols);
  const int64_t pruns = (rp + (256 >> lx) - 1) / (256 >> lx);
  const int64_t packs = std::min<int64_t>(std::max(64, 2048 / batch), pruns);
  const dim3 ngrid(parts, batch), pgrid(static_cast<unsigned>(packs), batch), block(256);
  const int64_t sx = static_cast<int64_t>(rp) * cp;
  if (vec) {
    hipLaunchKernelGGL((norm_kernel<T, true>), ngrid, block, 0, s, p, ldg, stride, rows, cols, lx, part);
    hipLaunchKernelGGL((pack_kernel<T, true>), pgrid, block, 0, s, p, ldg, stride, rows, cols, rp, cp, lx, part, parts,
                       steps, exps, hi, lo, sx);
  } else {
    hipLaunchKernelGGL((norm_kernel<T, false>), ngrid, block, 0, s, p, ldg, stride, rows, cols, lx, part);
    hipLaunchKernelGGL((pack_kernel<T, false>), pgrid, block, 0, s, p, ldg, stride, rows, cols, rp, cp, lx, part,
                       parts, steps, exps, hi, lo, sx);
  }
}

// Joins the ranges of k of A = X X^T (EPI_NS_PART, 64x64 tiles on and below the
// diagonal, item [matrix][range][tile]) in range order: a workgroup per 32x32
// block of a tile, stored on both sides of the diagonal.
__global__ void __launch_bounds__(256) gram_join_kernel(const float* __restrict__ part, int ranges, int tiles, int M,
                                                        float alpha, f16_t* __restrict__ hi, f16_t* __restrict__ lo,
                                                        int two, int64_t sa) {
  __shared__ float s[32][33];
  const int tile = blockIdx.x >> 2, sub = blockIdx.x & 3, b = blockIdx.y;
  int tm = static_cast<int>((sqrtf(8.f * tile + 1.f) - 1.f) * 0.5f);
  while (tm * (tm + 1) / 2 > tile) --tm;
  while ((tm + 1) * (tm + 2) / 2 <= tile) ++tm;
  const int tn = tile - tm * (tm + 1) / 2;
  const int r0 = (sub >> 1) * 32, c0 = (sub & 1) * 32;
  if (tm * 64 + r0 >= M || tn * 64 + c0 >= M) return;  // lengths are multiples of 32
  const int r = threadIdx.x >> 3, c = (threadIdx.x & 7) * 4;
  const float* p = part + (static_cast<int64_t>(b) * ranges * tiles + tile) * 4096 + (r0 + r) * 64 + c0 + c;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int k = 0; k < ranges; ++k) {
    const float4 x = *reinterpret_cast<const float4*>(p + static_cast<int64_t>(k) * tiles * 4096);
    v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
  }
  typedef _Float16 h4 __attribute__((ext_vector_type(4)));
  auto store = [&](int row, int col) {
    h4 a, l;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      a[k] = static_cast<_Float16>(v[k]);
      l[k] = static_cast<_Float16>(v[k] - static_cast<float>(a[k]));
    }
    const int64_t at = b * sa + static_cast<int64_t>(row) * M + col;
    *reinterpret_cast<h4*>(hi + at) = a;
    if (two) *reinterpret_cast<h4*>(lo + at) = l;
  };
#pragma unroll
  for (int k = 0; k < 4; ++k) s[r][c + k] = v[k] *= alpha;
  store(tm * 64 + r0 + r, tn * 64 + c0 + c);
  if (tm == tn) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = s[c + k][r];
  store(tn * 64 + c0 + r, tm * 64 + r0 + c);
}

// No steps: out from X itself.
template <typename TO, bool ACC>
__global__ void __launch_bounds__(256) unpack_kernel(const f16_t* __restrict__ hi, const f16_t* __restrict__ lo,
                                                     int64_t sx, int cp, const int* __restrict__ exps,
                                                     TO* __restrict__ out, int64_t ldo, int64_t so, int rows, int cols,
                                                     float scale, float keep) {
  const int64_t n = static_cast<int64_t>(rows) * cols;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = i / cols, c = i - row * cols, at = blockIdx.y * sx + row * cp + c;
    const float v = scale * ldexpf(static_cast<float>(hi[at]) + static_cast<float>(lo[at]), -exps[blockIdx.y * NS_EXPS]);
    TO* o = out + blockIdx.y * so + row * ldo + c;
    *o = ACC ? from_f<TO>(fmaf(keep, to_f<TO>(*o), v)) : from_f<TO>(v);
  }
}

inline uint64_t up(uint64_t n) { return (n + 255) & ~255ull; }

constexpr int CUS = 256;

// Tile of a product (0 A, 1 B, 2 X): the smallest predicted time.  A CU's k tile
// (32) takes `lat` us of one workgroup alone on it and `ktile` of each of
// several, a workgroup's start and epilogue `fixed`.  Fitted to 33 products of 256 to
// 20480 in one and three passes; B X reads and writes both planes of X, 8 bytes
// an entry that no product hides in 256x256 tiles (4096 x 4096: 25 of 130 us).
// 4096 x 4096, A: 192x192 tiles fill 253 CUs and take 78 us, 256x256 136 CUs and
// 91, 128x128 two or three to a CU and 107; 12 x 768 x 768, B X: 24 us in
// 128x128, 28 in 192x192, 40 in 256x256.
int tile_of(int product, int M, int N, int ktiles, int batch, double* us_out = nullptr) {
  struct {
    int bs;
    double lat, ktile, fixed[3];
  } const cfg[] = {{256, 0.74, 0.74, {8.0, 9.5, 20.0}}, {192, 0.45, 0.48, {9.0, 10.0, 11.0}},
                   {128, 0.30, 0.25, {2.5, 3.2, 4.0}}, {64, 0.147, 0.117, {0.8, 0.9, 0.7}}};
  int best = 0;
  double best_us = 0.0;
  for (const auto& c : cfg) {
    const int64_t tm = (M + c.bs - 1) / c.bs, tn = (N + c.bs - 1) / c.bs;
    const int64_t tiles = (product < 2 ? tm * (tm + 1) / 2 : tm * tn) * batch;
    const double share = static_cast<double>((tiles + CUS - 1) / CUS);
    const double us = ktiles * std::max(c.lat, share * c.ktile) + share * c.fixed[product];
    if (best == 0 || us < best_us) best = c.bs, best_us = us;
  }
  if (us_out) *us_out = best_us;
  return best;
}

// Ranges of k for A = X X^T of a short side M: 64x64 tiles in ranges and the
// joining kernel (4 us and its partial sums' way through memory) where that takes
// less time than the best tile alone, as with few tiles and a long k.
int ranges_of(int M, int ktiles, int batch) {
  double whole, best_us;
  tile_of(0, M, M, ktiles, batch, &whole);
  int best = 1;
  best_us = whole;
  const int64_t t = (M + 63) / 64, tiles = t * (t + 1) / 2 * batch;
  for (int n = 2; n <= 64; n *= 2) {
    if (ktiles < 8 * n || tiles * n > 4 * CUS) break;
    const double share = static_cast<double>((tiles * n + CUS - 1) / CUS), kt = static_cast<double>((ktiles + n - 1) / n);
    const double us = kt * std::max(0.147, share * 0.117) + share * 0.8 + 4.0 + tiles * n * 16384 * 2 / 4e6;
    if (us < best_us) best = n, best_us = us;
  }
  return best;
}


// Workspace: partial sums, X (hi and lo, each twice: a step reads one and
// writes the other; one plane's lo is read and written by the same lanes, so it
// is there once), A, B, and the sums of the ranges of k.
struct Ws {
  int rp, cp, k;  // padded lengths, the smaller of them
  int ranges;     // of k that A is the sum of
  uint64_t part, exps, x[2], xl[2], a, al, b, bl, sums, end;
};
// two: both planes of every factor (results in fp32).
Ws layout(bool two, int batch, int rows, int cols) {
  Ws w;
  w.rp = (rows + 31) / 32 * 32, w.cp = (cols + 31) / 32 * 32, w.k = std::min(w.rp, w.cp);
  const uint64_t x = up(2ull * batch * w.rp * w.cp), a = up(2ull * batch * w.k * w.k);
  uint64_t at = 0;
  auto take = [&](uint64_t n) { const uint64_t o = at; at += n; return o; };
  w.part = take(up(sizeof(double) * batch * norm_parts(batch, rows, cols)));
  w.exps = take(up(sizeof(int) * NS_EXPS * batch));
  w.x[0] = take(x);
  w.xl[0] = take(x);
  w.x[1] = take(x);
  w.xl[1] = two ? take(x) : w.xl[0];
  w.a = take(a);
  w.al = two ? take(a) : w.a;
  w.b = take(a);
  w.bl = two ? take(a) : w.b;
  w.ranges = ranges_of(w.k, (two ? 3 : 1) * std::max(w.rp, w.cp) / 32, batch);
  const uint64_t t = (w.k + 63) / 64;
  w.sums = take(w.ranges > 1 ? t * (t + 1) / 2 * w.ranges * batch * 4096 * 4 : 0);
  w.end = at;
  return w;
}

}  // namespace

// Tiles are counted in 32 bits, of 64 x 64 at least, and each is a workgroup.
bool orthogonalize_ok(int batch, int rows, int cols) {
  if (batch < 0 || rows <= 0 || cols <= 0 || batch > 65535 || rows > (1 << 24) || cols > (1 << 24)) return false;
  const int64_t tr = (rows + 63) / 64, tc = (cols + 63) / 64;
  if (batch == 0) return tr * tc < (1ll << 30);
  if (tr * tc * batch >= (1ll << 30) || std::min(tr, tc) * std::min(tr, tc) * batch >= (1ll << 30)) return false;
  for (const bool two : {false, true}) {
    const Ws o = layout(two, batch, rows, cols);
    const int passes = two ? 3 : 1, k = o.k / 32 * passes, n = std::max(o.rp, o.cp) / 32 * passes;
    auto fits = [&](int product, int M, int N, int ktiles) {
      const int bs = tile_of(product, M, N, ktiles, batch);
      const int64_t tm = (M + bs - 1) / bs, tn = (N + bs - 1) / bs;
      return (product < 2 ? tm * (tm + 1) / 2 : tm * tn) * batch < MAX_WORKGROUPS;
    };
    if (!fits(0, o.k, o.k, n) || !fits(1, o.k, o.k, k) || !fits(2, o.rp, o.cp, k)) return false;
  }
  return true;
}

// Coefficients whose steps keep the singular values, which start in [0, 1], and
// the entries of b A + c A^2 in fp16's range: bounds of s <- |a s + b s^3 + c
// s^5| and |b t + c t^2|, t = s^2, from their extrema.
bool orthogonalize_coef_ok(const float* coef, int steps) {
  double top = 1.0;
  for (int k = 0; k < steps; ++k) {
    const double a = coef[3 * k], b = coef[3 * k + 1], c = coef[3 * k + 2];
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    const double t = top * top;
    auto p = [&](double x) { return std::fabs(b * x + c * x * x); };
    double poly = p(t);
    if (c != 0.0 && -b / (2 * c) > 0.0 && -b / (2 * c) < t) poly = std::max(poly, p(-b / (2 * c)));
    top = step_bound(a, b, c, top);
    if (poly > 32.0 || top > 4.0 || std::fabs(a) > 32.0) return false;
  }
  return true;
}

// Enough for either type of result.
uint64_t orthogonalize_ws(int batch, int rows, int cols) {
  return std::max(layout(false, batch, rows, cols).end, layout(true, batch, rows, cols).end);
}

hipError_t orthogonalize(int dtype, const void* g, int64_t ldg, int64_t stride_g, void* out, int64_t ldo,
                         int64_t stride_o, int out_epi, float keep, float scale, int batch, int rows, int cols,
                         const float* coef, int steps, void* ws, hipStream_t s) {
  const int out_mode = out_epi == EPI_ACC_F32 ? 2 : out_epi == EPI_STORE_F32 || dtype == DT_F32 ? 1 : 0;
  const bool two = out_mode != 0;  // of an fp32 result every factor has both planes
  const Ws o = layout(two, batch, rows, cols);
  char* base = static_cast<char*>(ws);
  auto at = [&](uint64_t off) { return reinterpret_cast<f16_t*>(base + off); };
  const int64_t sx = static_cast<int64_t>(o.rp) * o.cp, sa = static_cast<int64_t>(o.k) * o.k;
  double* part = reinterpret_cast<double*>(base + o.part);
  int* exps = reinterpret_cast<int*>(base + o.exps);
  const int64_t n = static_cast<int64_t>(rows) * cols;
  Steps st{};
  st.n = steps;
  double r = 1.0;
  for (int k = 0; k < steps; ++k) {
    for (int i = 0; i < 3; ++i) st.coef[3 * k + i] = coef[3 * k + i];
    st.exps[k] = exponent_of(r);
    r = step_bound(coef[3 * k], coef[3 * k + 1], coef[3 * k + 2], r);
  }
  if (dtype == DT_BF16)
    launch_pack<bf16_t>(g, ldg, stride_g, batch, rows, cols, o.rp, o.cp, part, st, exps, at(o.x[0]), at(o.xl[0]), s);
  else
    launch_pack<float>(g, ldg, stride_g, batch, rows, cols, o.rp, o.cp, part, st, exps, at(o.x[0]), at(o.xl[0]), s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  scale /= SCALE;
  if (steps == 0) {
    const dim3 ugrid(static_cast<unsigned>(std::min<int64_t>((n + 255) / 256, 2048)), batch);
#define ATOM_UNPACK(TO, ACC)                                                                                     \
  hipLaunchKernelGGL((unpack_kernel<TO, ACC>), ugrid, dim3(256), 0, s, at(o.x[0]), at(o.xl[0]), sx, o.cp, exps,  \
                     static_cast<TO*>(out), ldo, stride_o, rows, cols, scale, keep)
    if (out_mode == 0) ATOM_UNPACK(bf16_t, false);
    else if (out_mode == 1) ATOM_UNPACK(float, false);
    else ATOM_UNPACK(float, true);
#undef ATOM_UNPACK
    return hipGetLastError();
  }
  const bool wide = rows <= cols;
  const int planes = two ? 2 : 1, passes = two ? 3 : 1;
  const int osz = out_mode == 0 ? 2 : 4;
  for (int k = 0; k < steps; ++k) {
    const int i = k & 1;
    const float a = coef[3 * k], b = coef[3 * k + 1], c = coef[3 * k + 2];
    auto product = [&](GemmArgs& p, int len, bool akc, bool bkc, int epi) {
      p.ns.kp = len / 32;
      p.K = passes * len;
      p.splits = 1;
      return gemm_ns(p, tile_of(epi - EPI_NS_GRAM, p.M, p.N, passes * p.ns.kp, batch), planes, batch, akc, bkc, epi, s);
    };
    GemmArgs p{};
    p.A = p.B = at(o.x[i]), p.lda = p.ldb = o.cp, p.C = at(o.a), p.ldc = o.k;
    p.M = p.N = o.k;
    p.alpha = 1.f / SCALE;
    p.ns.sa = p.ns.sb = sx, p.ns.sc = sa;
    p.ns.pa = p.ns.pb = at(o.xl[i]) - at(o.x[i]);
    p.ns.C_lo = at(o.al);
    if (o.ranges > 1) {
      const int len = wide ? o.cp : o.rp;
      p.ns.kp = len / 32;
      p.K = passes * len;
      p.splits = 1;
      p.C = base + o.sums;
      p.ns.range = (passes * p.ns.kp + o.ranges - 1) / o.ranges;
      p.ns.ranges = (passes * p.ns.kp + p.ns.range - 1) / p.ns.range;  // none empty
      e = gemm_ns(p, 64, planes, batch, wide, wide, EPI_NS_PART, s);
      if (e != hipSuccess) return e;
      const int t = (o.k + 63) / 64, tiles = t * (t + 1) / 2;
      hipLaunchKernelGGL(gram_join_kernel, dim3(4 * tiles, batch), dim3(256), 0, s, reinterpret_cast<float*>(base + o.sums),
                         p.ns.ranges, tiles, o.k, 1.f / SCALE, at(o.a), at(o.al), two ? 1 : 0, sa);
      e = hipGetLastError();
    } else {
      e = product(p, wide ? o.cp : o.rp, wide, wide, EPI_NS_GRAM);
    }
    if (e != hipSuccess) return e;
    GemmArgs q{};
    q.A = q.B = at(o.a), q.lda = q.ldb = o.k, q.C = at(o.b), q.ldc = o.k;
    q.M = q.N = o.k;
    q.alpha = c / SCALE;
    q.ns.sa = q.ns.sb = q.ns.sc = sa;
    q.ns.pa = q.ns.pb = at(o.al) - at(o.a);
    q.ns.aux = at(o.a), q.ns.aux_lo = at(o.al), q.ns.beta = b, q.ns.C_lo = at(o.bl);
    q.ns.exps = exps + k;
    e = product(q, o.k, true, true, EPI_NS_POLY);
    if (e != hipSuccess) return e;
    GemmArgs r{};
    r.A = wide ? at(o.b) : at(o.x[i]), r.B = wide ? at(o.x[i]) : at(o.b);
    r.lda = wide ? o.k : o.cp, r.ldb = wide ? o.cp : o.k;
    r.C = at(o.x[1 - i]), r.ldc = o.cp;
    r.M = o.rp, r.N = o.cp;
    r.alpha = 1.f / SCALE;
    r.ns.sa = wide ? sa : sx, r.ns.sb = wide ? sx : sa, r.ns.sc = sx;
    r.ns.pa = wide ? at(o.bl) - at(o.b) : at(o.xl[i]) - at(o.x[i]);
    r.ns.pb = wide ? at(o.xl[i]) - at(o.x[i]) : at(o.bl) - at(o.b);
    r.ns.aux = at(o.x[i]), r.ns.aux_lo = at(o.xl[i]), r.ns.beta = a, r.ns.C_lo = at(o.xl[1 - i]);
    r.ns.exps = exps + k;
    r.ns.out_mode = 3;
    if (k == steps - 1) {
      r.ns.out = out, r.ns.ldo = ldo, r.ns.so = stride_o, r.ns.out_mode = out_mode;
      r.ns.orows = rows, r.ns.ocols = cols, r.ns.scale = scale, r.ns.keep = keep;
      r.ns.vec = cols % 4 == 0 && ldo % 4 == 0 && stride_o % 4 == 0 && reinterpret_cast<uintptr_t>(out) % (4 * osz) == 0;
    }
    e = product(r, o.k, true, !wide, EPI_NS_STEP);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace atom

// Tiles of a step's three products and ranges of k of the first, by the type of
// the result (tests).
extern "C" void atom_ns_choice(int dtype, int batch, int rows, int cols, int* out) {
  using namespace atom;
  const Ws o = layout(dtype == DT_F32, batch, rows, cols);
  const int passes = dtype == DT_F32 ? 3 : 1, lng = std::max(o.rp, o.cp);
  out[0] = tile_of(0, o.k, o.k, passes * lng / 32, batch);
  out[1] = tile_of(1, o.k, o.k, passes * o.k / 32, batch);
  out[2] = tile_of(2, o.rp, o.cp, passes * o.k / 32, batch);
  out[3] = o.ranges;
}
