// What the cross-attention kernels (cross_attention.hip, bf16;
// cross_attention_f32.hip) and their launcher share: the arguments, a
// sequence's rows, the mapping of workgroups, and the kernels that join ranges.
//
// A sequence's queries of the G heads that share a head of keys are packed into
// one list of rows, p = t G + g: one token of many heads still fills the rows of
// a matrix instruction, and the shared keys are read once for all of them.
#pragma once

#include "attention_kernels.h"

namespace atom {

namespace cross {

// A sequence's rows: the first, and how many.  Lengths and starts are clamped
// to the buffer, so no value of them leads out of it.
struct Seq {
  int64_t row0;
  int n;
};
ATOM_DEV Seq seq(const int32_t* start, const int32_t* len, int T, int64_t rows, int b) {
  int n = len ? min(max(len[b], 0), T) : T;
  if (!start) return Seq{static_cast<int64_t>(b) * T, n};
  const int64_t r = start[b];
  if (r < 0 || r >= rows) return Seq{0, 0};
  return Seq{r, static_cast<int>(min(static_cast<int64_t>(n), rows - r))};
}

// Work item of a workgroup: the hardware hands consecutive ids to the eight XCDs
// in turn; each XCD takes a run of consecutive items, so that the blocks of one
// sequence and head, which read the same keys, share an L2.  Heads are outside,
// sequences inside (bh = head B + sequence), so that every XCD has some of the
// long and some of the short sequences.  Ids past the items
// (the grid is a multiple of eight) are negative.
ATOM_DEV int item_of(int n_items, int id) {
  const int per = (n_items + 7) >> 3;
  const int i = (id & 7) * per + (id >> 3);
  return (id >> 3) < per && i < n_items ? i : -1;
}

// Token and head (of the group) of packed row p.
struct Row {
  int t, g;
};
ATOM_DEV Row row_of(const CrossArgs& a, int p) {
  if (a.G == 1) return Row{p, 0};
  const int t = static_cast<int>(__umulhi(static_cast<uint32_t>(p), a.gmul));
  return Row{t, p - t * a.G};
}

// Offset of packed row p of head group hk in a tensor of leading dimension ld.
template <int DH>
ATOM_DEV int64_t at(const CrossArgs& a, const Seq& s, int hk, int p, int64_t ld) {
  const Row r = row_of(a, p);
  return (s.row0 + r.t) * ld + static_cast<int64_t>(hk * a.G + r.g) * DH;
}

// log-sum-exp for the backward's exponents (in base 2): a row that has none (no
// finite score) gets +infinity, and so no weight anywhere.
ATOM_DEV float lse_of(float lse) { return lse == -INFINITY ? INFINITY : lse; }
ATOM_DEV float lse2_of(float lse) { return lse_of(lse) * attn::LOG2E; }

// Queries whose D fits beside the stages of a small backward's workgroup.
constexpr int SMALL_ROWS = 2048;

// Where the running maximum starts: below every finite score, and finite, so
// that a score of -infinity weighs 0 against it.
constexpr float NO_MAX = -3e38f;

// e^t for t <= 0 to an fp32 rounding or two: the part of t log2(e) that fp32 cuts
// off goes into the result (with it cut, p is off by |t| 2^-24: at lse 8, 1e-6).
// The fp32 kernels keep maxima and lse in natural units.
ATOM_DEV float exp_near(float t) {
  const float h = t * attn::LOG2E, r = __builtin_fmaf(t, attn::LOG2E, -h) + t * 1.92596299e-8f;
  const float p = attn::ex2(h);
  return t < -104.f ? 0.f : __builtin_fmaf(p, r * attn::LN2, p);
}

// A row's output from the sums of its ranges: W waves a row, each with every W-th
// range in order, then the waves in order.  A lane takes the weight of one range in
// 64, the wave their sums, eight loads in flight.
template <typename T, int DH, int W>
__global__ void __launch_bounds__(W == 1 ? 256 : 64 * W) cross_join_kernel(const CrossArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t P = static_cast<int64_t>(a.Tq) * a.G, n = P * a.B * a.Hk;
  const int64_t r = W == 1 ? static_cast<int64_t>(blockIdx.x) * 4 + wave : blockIdx.x;
  const int first = W == 1 ? 0 : wave;
  if (r >= n) return;
  const int bh = static_cast<int>(r / P), p = static_cast<int>(r % P), b = bh % a.B, hk = bh / a.B;
  const Seq qs = seq(a.q_start, a.q_len, a.Tq, a.q_rows, b);
  const bool on = p < qs.n * a.G;
  if (!on && a.q_start) return;
  constexpr int E = DH / 64;
  constexpr bool NATURAL = sizeof(T) == 4;  // the maxima's units
  float m = NO_MAX, l = 0.f, o[E] = {};
  if (on) {
    for (int s = lane; s < a.splits; s += 64) m = fmaxf(m, a.ml[2 * (s * n + r)]);
    m = wave_max(m);
    for (int s0 = first; s0 < a.splits; s0 += 64 * W) {
      const int s = s0 + lane * W, count = min(64, (a.splits - s0 + W - 1) / W);
      float f = 0.f;
      if (s < a.splits) {
        const float t = a.ml[2 * (s * n + r)] - m;
        f = NATURAL ? exp_near(t) : attn::ex2(t);
        l += f * a.ml[2 * (s * n + r) + 1];
      }
      const float* part = a.part + (s0 * n + r) * DH + E * lane;
      for (int i0 = 0; i0 < count; i0 += 8) {
        float v[8][E];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < E; ++e) v[i][e] = part[min(i0 + i, count - 1) * (W * n * DH) + e];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (i0 + i >= count) break;
          const float fi = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), i0 + i));
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] += fi * v[i][e];
        }
      }
    }
    l = wave_sum(l);
  }
  if constexpr (W > 1) {
    __shared__ float sums[W][64][E + 1];
#pragma unroll
    for (int e = 0; e < E; ++e) sums[wave][lane][e] = o[e];
    sums[wave][lane][E] = l;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < W; ++w) {
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] += sums[w][lane][e];
      l += sums[w][lane][E];
    }
  }
  const int64_t lo = at<DH>(a, qs, hk, p, a.ldo) + E * lane;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) static_cast<T*>(a.o)[lo + e] = from_f<T>(o[e] * inv);
  if (a.lse && lane == 0) {
    const Row w = row_of(a, p);
    a.lse[(qs.row0 + w.t) * a.Hq + hk * a.G + w.g] = l == 0.f ? -INFINITY : NATURAL ? m + logf(l) : (m + log2f(l)) * attn::LN2;
  }
}

}  // namespace cross

hipError_t cross_fwd_f32(const CrossArgs& a, int dh, hipStream_t s);
hipError_t cross_bwd_f32(const CrossArgs& a, int dh, bool small, hipStream_t s);

}  // namespace atom
