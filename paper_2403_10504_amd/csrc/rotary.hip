// Rotary positions, and norms of queries and keys with the rotation in the same
// pass (atom_k_rope, atom_k_qknorm_rope_fwd, _bwd).
//
// Pair i of a head at position p turns by a = p freq_i:
//   (u, w) -> m (u cos a - w sin a, u sin a + w cos a);
// the transposed turn (its gradient) has -a.  The norm is u = g x r with
// r = 1/sqrt(mean x^2 + eps), in front of the turn.  With g' the gradient turned
// back, its own gradient is
//   dg = sum over rows and heads of g' x r,   dx = r (g' g - x r mean(g' g x r)).
//
// The kernels are bound by memory: each head is read once and written once
// (the norm's backward: dy and x once, dx once; r is computed again rather than
// kept, the whole head being in registers anyway).  4096 rows of 3 x 32 heads of 128:
// 39 us, 5.2 TB/s (a large copy: 5.1); gradients of 2048 rows of 3 x 40: 35 us, 4.8
// TB/s, and 4 for the gains' sums; queries and keys of 8192 rows of 16 heads turned:
// 29.8 us, 4.5 TB/s.  Where head, rot or a pitch allows less than 16 bytes an access
// (pairs_of), less: 4096 rows of 3 x 32 heads of 128, bf16, 41 us in 16 bytes, 48 in 8,
// 61 in 4, 95 in 2; fp32, 2048 rows, 45, 61 and 94 in 16, 8 and 4; heads of 130 123 and
// 112; gradients, 2048 rows bf16, 32, 45, 64 and 83.
//
// A lane holds V pairs of a head: in the half layout V elements at c V and V at
// rot/2 + c V, in the pairs layout 2 V in a row; elements past rot in chunks of
// 2 V, which do not turn.  So a pair never leaves its lane, P lanes (a power of
// two) hold a head, and a wave 64 / P heads at a time.  A wave takes a whole
// row, so the angles of its V pairs, and their sines, are computed once for all
// of the row's heads; where rows are few a row's heads go to several waves, where a
// row's heads are few several rows to one.
//
// Sines are computed one a lane and passed on through LDS inside the wave: they are
// the same in every head, and a lane alone would compute V of them.
//
// Angles are computed in 64 bits, with what those round off kept (half_turns): p
// freq_i in fp32 is off by a whole turn's part from p = 10^5 on (2^-24 of 10^5
// radians: 0.006).
#include <math.h>

#include <algorithm>

#include "../../include/atom.h"
#include "../../include/atom_kernels.h"
#include "common.h"
#include "launch.h"

namespace atom {
namespace {

constexpr int WAVES = 4;  // waves of a workgroup

struct Args {
  const void* x;
  const void* dy;  // backward
  void* y;         // y, or dx
  int64_t ldx, lddy, ldy;
  const void *gq, *gk;  // gains, null: 1
  float* part;          // backward: [workgroups][2][dh] partial sums of the gains' gradients, null: not wanted
  const int32_t* pos;   // null: row % T
  const double* freq;
  float mscale, eps;
  int back;     // rope: the transposed turn
  uint32_t rows, T;
  int Hq, Hk, Hv;  // (rope: Hq alone)
  int dh, rot;
  int plog, rlog;  // log2 of P, and of the rows that a wave takes at a time
  int per;         // groups of heads that a workgroup takes of a row
  int copy;        // the value heads are copied
};

enum { ROPE, NORM, NORM_BWD };

// V elements, in one load of up to 16 bytes
template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
  T e[V];
};

// A lane's two runs of V elements of a head, as they are in memory.  Inputs are
// read once, past the caches' order of use (norm_6.7b 44.6 -> 39.7 us, norm_grad_13b
// 46.9 -> 38.5); results are stored the ordinary way: the attention behind finds
// them in the Infinity Cache (norm and causal attention at 8 x 2048, 12 heads of
// 64: 97.6 us, with streamed stores 103.5, the norm alone 33.7 and 24.2).
template <typename T, int V>
struct Raw {
  Vec<T, V> a, b;
  ATOM_DEV void load(const T* p, int o0, int o1) {
    a = one(p + o0);
    b = one(p + o1);
  }
  static ATOM_DEV Vec<T, V> one(const T* p) {
    if constexpr (sizeof(Vec<T, V>) == 16) {
      typedef uint32_t u4 __attribute__((ext_vector_type(4)));
      return __builtin_bit_cast(Vec<T, V>, __builtin_nontemporal_load(reinterpret_cast<const u4*>(p)));
    } else {
      return *reinterpret_cast<const Vec<T, V>*>(p);
    }
  }
  ATOM_DEV void store(T* p, int o0, int o1) const {
    *reinterpret_cast<Vec<T, V>*>(p + o0) = a;
    *reinterpret_cast<Vec<T, V>*>(p + o1) = b;
  }
};

// The same as pairs (u, w).
template <typename T, int V, bool PAIRS>
struct Chunk {
  float u[V], w[V];
  ATOM_DEV void set(const Raw<T, V>& r) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if constexpr (PAIRS) {
        const int e = 2 * i;
        u[i] = to_f<T>(e < V ? r.a.e[e % V] : r.b.e[e % V]);
        w[i] = to_f<T>(e + 1 < V ? r.a.e[(e + 1) % V] : r.b.e[(e + 1) % V]);
      } else {
        u[i] = to_f<T>(r.a.e[i]);
        w[i] = to_f<T>(r.b.e[i]);
      }
    }
  }
  ATOM_DEV Raw<T, V> get() const {
    Raw<T, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if constexpr (PAIRS) {
        r.a.e[i] = from_f<T>(i % 2 ? w[i / 2] : u[i / 2]);
        r.b.e[i] = from_f<T>((V + i) % 2 ? w[(V + i) / 2] : u[(V + i) / 2]);
      } else {
        r.a.e[i] = from_f<T>(u[i]);
        r.b.e[i] = from_f<T>(w[i]);
      }
    }
    return r;
  }
};

// v of another lane of the row of 16, by data-parallel-primitive control word.
template <int CTRL>
ATOM_DEV float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// The sum over P neighbouring lanes, in all of them: pairs, quads (quad_perm),
// then halves and rows of equal values, mirrored, then rows against each other.
ATOM_DEV float sum_inside(float v, int P) {
  float a, b;
  if (P > 1) v += dpp<0xB1>(v);
  if (P > 2) v += dpp<0x4E>(v);
  if (P > 4) v += dpp<0x141>(v);
  if (P > 8) v += dpp<0x140>(v);
  if (P > 16) pair16(v, a, b), v = a + b;
  if (P > 32) pair32(v, a, b), v = a + b;
  return v;
}

// p freq / pi, less the whole turns, to 2^-25 (fp32's half step below 1): what the
// products with 1/pi (in two doubles) and with p round off is added behind the
// reduction, which is exact.  (Rounded to 64 bits alone, angles of 2 10^9 radians are
// off by up to 5 10^-7.)  Not contracted: in a fused product t would not be the value
// that its rest was taken of.
ATOM_DEV float half_turns(double p, double freq) {
#pragma clang fp contract(off)
  constexpr double INV_PI = 0x1.45f306dc9c883p-2, INV_PI_LOW = -0x1.6b01ec5417056p-56;
  const double q = freq * INV_PI, q_low = __builtin_fma(freq, INV_PI, -q) + freq * INV_PI_LOW;
  const double t = p * q, t_low = __builtin_fma(p, q, -t) + p * q_low;
  const double rest = (t - 2.0 * rint(0.5 * t)) + t_low;
  return static_cast<float>(rest - 2.0 * rint(0.5 * rest));  // (beyond 1 fp32's step is twice as long)
}

// NC chunks of a lane (two for heads of more than 128 elements in single pairs).
// (Waves a SIMD: the norms within 128 registers 44.6 us, 135 unbounded 47.0, 96 48;
// the gradients within 168 49.3, within 256 48.8, 128 spill: 92.)
// MIX: groups of several sides (kind_of), and several rows a wave.
template <typename T, int V, int NC, bool PAIRS, int OP, bool MIX>
__global__ void __launch_bounds__(64 * WAVES, OP == NORM_BWD ? 2 : 4) rotary_kernel(const Args a) {
  using C = Chunk<T, V, PAIRS>;
  using R = Raw<T, V>;
  constexpr int PAIRS_MAX = MIX ? 64 * V : 128;  // (64 lanes of V pairs; a row has 128 at most)
  __shared__ float2 turns[WAVES][PAIRS_MAX];       // cosine and sine of the rows' pairs, times mscale
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int P = 1 << a.plog, rlog = MIX ? a.rlog : 0, slog = 6 - a.plog - rlog, S = 1 << slog;
  const int lp = lane & (P - 1), slot = (lane >> a.plog) & (S - 1), ri = MIX ? lane >> (a.plog + slog) : 0;
  const int L = a.dh / (2 * V), rc = a.rot / (2 * V);
  const float inv_dh = 1.f / a.dh;
  int o0[NC], o1[NC];
  bool on[NC], turn[NC];
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const int c = lp + 64 * k;
    on[k] = c < L;
    turn[k] = c < rc;
    if (!turn[k] || PAIRS) o0[k] = 2 * V * c, o1[k] = o0[k] + V;
    else o0[k] = V * c, o1[k] = a.rot / 2 + V * c;
  }
  const int Hq = a.Hq, Hk = a.Hk, Hv = a.copy ? a.Hv : 0, H = Hq + Hk + Hv;
  const int gq = (Hq + S - 1) >> slog, gk = (Hk + S - 1) >> slog, gv = (Hv + S - 1) >> slog;
  const int g0 = blockIdx.y * a.per, g1 = min(g0 + a.per, MIX ? (H + S - 1) >> slog : gq + gk + gv);

  C gain[NC];
  float acc[2][NC][2 * V];  // of queries and of keys
  if constexpr (OP == NORM_BWD) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) acc[s][k][i] = 0.f;
  }
  auto load_gain = [&](const void* g) {
#pragma unroll
    for (int k = 0; k < NC; ++k) {
#pragma unroll
      for (int i = 0; i < V; ++i) gain[k].u[i] = gain[k].w[i] = 1.f;
      if (g && on[k]) {
        R r;
        r.load(static_cast<const T*>(g), o0[k], o1[k]);
        gain[k].set(r);
      }
    }
  };
  // Group g: what its heads are (ALL_Q, ALL_K, ALL_V, or g itself if of several
  // sides), and the lane's head.
  enum { ALL_Q = -1, ALL_K = -2, ALL_V = -3 };
  auto kind_of = [&](int g) -> int {
    if (!MIX) return g < gq ? ALL_Q : g < gq + gk ? ALL_K : ALL_V;
    const int first = g << slog, last = min(first + S, H) - 1;
    return last < Hq ? ALL_Q : first >= Hq + Hk ? ALL_V : first >= Hq && last < Hq + Hk ? ALL_K : g;
  };
  struct Head {
    bool is_q, is_v, there;
    int at;  // of its first element in the row (2^16 heads of 256 at most)
  };
  bool row_there = true;
  // (by value: between variables captured by reference the compiler selects an
  // address, which puts them in memory)
  auto head_at = [](int g, int slog, int slot, int gq, int gk, int Hq, int Hk, int Hv, int dh, bool row_there) {
    if (MIX) {
      const int i = (g << slog) + slot;
      return Head{i < Hq, i >= Hq + Hk, i < Hq + Hk + Hv && row_there, i * dh};
    }
    const bool is_q = OP == ROPE || g < gq, is_v = OP != ROPE && g >= gq + gk;
    const int i = ((is_q ? g : is_v ? g - gq - gk : g - gq) << slog) + slot;
    return Head{is_q, is_v, i < (is_q ? Hq : is_v ? Hv : Hk), (is_q ? i : is_v ? Hq + Hk + i : Hq + i) * dh};
  };
  auto head_of = [&](int g) { return head_at(g, slog, slot, gq, gk, Hq, Hk, Hv, a.dh, row_there); };
  // (several rows are within 2^31 elements)
  const int rx_off = MIX ? ri * static_cast<int>(a.ldx) : 0, rd_off = MIX ? ri * static_cast<int>(a.lddy) : 0;
  const int ry_off = MIX ? ri * static_cast<int>(a.ldy) : 0;

  for (uint64_t row = (static_cast<uint64_t>(blockIdx.x) * WAVES + wave) << rlog; row < a.rows;
       row += static_cast<uint64_t>(gridDim.x) * WAVES << rlog) {
    if (MIX) row_there = row + ri < a.rows;
    const T* x = static_cast<const T*>(a.x) + static_cast<int64_t>(row) * a.ldx;
    const T* dy = OP == NORM_BWD ? static_cast<const T*>(a.dy) + static_cast<int64_t>(row) * a.lddy : x;
    T* y = static_cast<T*>(a.y) + static_cast<int64_t>(row) * a.ldy;
    // the next group's loads are in flight while one is worked on, the first
    // one's while the angles are computed
    R rx[NC], rd[NC];
    auto fetch = [&](const Head& h) {
#pragma unroll
      for (int k = 0; k < NC; ++k) {
#pragma unroll
        for (int i = 0; i < V; ++i) rx[k].a.e[i] = rx[k].b.e[i] = rd[k].a.e[i] = rd[k].b.e[i] = 0;
        if (h.there && on[k]) {
          if (OP == NORM_BWD) rd[k].load(dy + rd_off + h.at, o0[k], o1[k]);
          if (OP != NORM_BWD || !h.is_v) rx[k].load(x + rx_off + h.at, o0[k], o1[k]);
        }
      }
    };
    Head h = head_of(g0);
    fetch(h);
    float cs[NC][V], sn[NC][V];
    if (a.rot) {
      // each lane one pair in 64 (they are the same in every head), passed on
      // through LDS inside the wave
      const int half = a.rot / 2, inv = (0x10000 + half - 1) / half;  // (i inv >> 16 is i / half below 512)
      const uint32_t t0 = a.pos ? 0 : static_cast<uint32_t>(row) % a.T;
      double p = 0.0;
      if (!MIX) p = a.pos ? static_cast<double>(a.pos[row]) : static_cast<double>(t0);
      for (int i = lane; i < half << rlog; i += 64) {
        const int r = MIX ? i * inv >> 16 : 0, pair = i - r * half;
        if (MIX && !a.pos) {
          uint32_t t = t0 + r;
          while (t >= a.T) t -= a.T;
          p = static_cast<double>(t);
        } else if (MIX && row + r < a.rows) {
          p = static_cast<double>(a.pos[row + r]);
        }
        float s, c;
        sincospif(half_turns(p, a.freq[pair]), &s, &c);
        turns[wave][i] = make_float2(c * a.mscale, (OP == NORM_BWD || (OP == ROPE && a.back) ? -s : s) * a.mscale);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int k = 0; k < NC; ++k)
        if (turn[k]) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float2 t = turns[wave][(MIX ? ri * (a.rot / 2) : 0) + V * (lp + 64 * k) + i];
            cs[k][i] = t.x;
            sn[k][i] = t.y;
          }
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    auto rotate = [&](C (&v)[NC]) {
#pragma unroll
      for (int k = 0; k < NC; ++k)
        if (turn[k]) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float u = v[k].u[i], w = v[k].w[i];
            // one order of roundings, whatever the width of the accesses
            v[k].u[i] = __builtin_fmaf(u, cs[k][i], -(w * sn[k][i]));
            v[k].w[i] = __builtin_fmaf(u, sn[k][i], w * cs[k][i]);
          }
        }
    };
    for (int g = g0; g < g1; ++g) {
      const Head cur = h;
      R cx[NC], cd[NC];
#pragma unroll
      for (int k = 0; k < NC; ++k) cx[k] = rx[k], cd[k] = rd[k];
      if (g + 1 < g1) {
        h = head_of(g + 1);
        fetch(h);
      }
      const int kind = OP == ROPE ? ALL_Q : kind_of(g);
      auto copy = [&] {  // values: as they are
#pragma unroll
        for (int k = 0; k < NC; ++k)
          if (cur.there && on[k]) (OP == NORM_BWD ? cd[k] : cx[k]).store(y + ry_off + cur.at, o0[k], o1[k]);
      };
      if (kind == ALL_V) {
        copy();
        continue;
      }
      if (OP != ROPE && (MIX || g == g0 || g == gq)) load_gain(cur.is_q ? a.gq : a.gk);
      C v[NC];
#pragma unroll
      for (int k = 0; k < NC; ++k) v[k].set(cx[k]);
      if constexpr (OP == ROPE) {
        rotate(v);
      } else {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NC; ++k)
#pragma unroll
          for (int i = 0; i < V; ++i) s += v[k].u[i] * v[k].u[i] + v[k].w[i] * v[k].w[i];
        const float r = __builtin_amdgcn_rsqf(sum_inside(s, P) * inv_dh + a.eps);
        if constexpr (OP == NORM) {
#pragma unroll
          for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
              v[k].u[i] *= r * gain[k].u[i];
              v[k].w[i] *= r * gain[k].w[i];
            }
          rotate(v);
        } else {
          C d[NC];
#pragma unroll
          for (int k = 0; k < NC; ++k) {
            d[k].set(cd[k]);
            if (MIX && kind >= 0) {  // (values add nothing to the gains, whatever they are)
#pragma unroll
              for (int i = 0; i < V; ++i) {
                d[k].u[i] = cur.is_v ? 0.f : d[k].u[i];
                d[k].w[i] = cur.is_v ? 0.f : d[k].w[i];
              }
            }
          }
          rotate(d);
          float m = 0.f;
#pragma unroll
          for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
              v[k].u[i] *= r;
              v[k].w[i] *= r;
              const float tu = d[k].u[i] * v[k].u[i], tw = d[k].w[i] * v[k].w[i];
              if (MIX) {
                if (kind != ALL_K) acc[0][k][2 * i] += cur.is_q ? tu : 0.f, acc[0][k][2 * i + 1] += cur.is_q ? tw : 0.f;
                if (kind != ALL_Q) acc[1][k][2 * i] += cur.is_q ? 0.f : tu, acc[1][k][2 * i + 1] += cur.is_q ? 0.f : tw;
              } else {
                if (cur.is_q) acc[0][k][2 * i] += tu, acc[0][k][2 * i + 1] += tw;
                else acc[1][k][2 * i] += tu, acc[1][k][2 * i + 1] += tw;
              }
              m += tu * gain[k].u[i] + tw * gain[k].w[i];
            }
          m = sum_inside(m, P) * inv_dh;
#pragma unroll
          for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
              v[k].u[i] = r * (d[k].u[i] * gain[k].u[i] - v[k].u[i] * m);
              v[k].w[i] = r * (d[k].w[i] * gain[k].w[i] - v[k].w[i] * m);
            }
        }
      }
#pragma unroll
      for (int k = 0; k < NC; ++k)
        if (cur.there && on[k] && !(MIX && kind >= 0 && cur.is_v)) v[k].get().store(y + ry_off + cur.at, o0[k], o1[k]);
      if (MIX && kind >= 0 && cur.is_v) copy();
    }
  }

  if constexpr (OP == NORM_BWD) {
    if (!a.part) return;
    // over the wave's slots (lanes P apart), then over the waves, in this order
    auto each = [&](auto f) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int k = 0; k < NC; ++k)
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) acc[s][k][i] = f(acc[s][k][i]);
    };
    if (P <= 1) each([](float v) { return v + dpp<0x121>(v); });  // (rotations of a row of 16)
    if (P <= 2) each([](float v) { return v + dpp<0x122>(v); });
    if (P <= 4) each([](float v) { return v + dpp<0x124>(v); });
    if (P <= 8) each([](float v) { return v + dpp<0x128>(v); });
    if (P <= 16)
      each([](float v) {
        float p, q;
        pair16(v, p, q);
        return p + q;
      });
    if (P <= 32)
      each([](float v) {
        float p, q;
        pair32(v, p, q);
        return p + q;
      });
    __shared__ float sums[WAVES][2][256];
    if (lane < P) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int k = 0; k < NC; ++k)
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) {
            // element i of the chunk: pair i / 2, first or second of it
            const int e = PAIRS ? i : (i & 1) * V + (i >> 1);
            if (on[k]) sums[wave][s][(e < V ? o0[k] + e : o1[k] + e - V)] = acc[s][k][i];
          }
    }
    __syncthreads();
    float* out = a.part + (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * 2 * a.dh;
    for (int t = threadIdx.x; t < 2 * a.dh; t += 64 * WAVES) {
      const int s = t >= a.dh, e = t - s * a.dh;
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v += sums[w][s][e];
      out[t] = v;
    }
  }
}

// dgq and dgk (null: not wanted) from the workgroups' sums [n][2][dh]: 16 columns
// of a workgroup, part slice, slice + 64, ... to each of 64 slices, then the
// slices in order.
__global__ void __launch_bounds__(1024) gain_sum_kernel(const float* __restrict__ part, int n, int dh, float* dgq,
                                                        float* dgk) {
  __shared__ float sh[64][16];
  const int cl = threadIdx.x & 15, sl = threadIdx.x >> 4, c = blockIdx.x * 16 + cl;
  float s = 0.f;
  if (c < 2 * dh) {
#pragma unroll 8
    for (int p = sl; p < n; p += 64) s += part[static_cast<int64_t>(p) * 2 * dh + c];
  }
  sh[sl][cl] = s;
  __syncthreads();
  for (int half = 32; half; half >>= 1) {
    if (sl < half) sh[sl][cl] += sh[sl + half][cl];
    __syncthreads();
  }
  float* out = c < dh ? dgq : dgk;
  if (sl == 0 && c < 2 * dh && out) out[c < dh ? c : c - dh] = sh[0][cl];
}

// The grid: workgroups of four rows, and the parts of a row's heads.
struct Shape {
  int per;
  unsigned gx, gy;
};

// Pairs in a lane: as many as 16-byte accesses, the layout of the head and the
// alignment of every buffer allow.
int pairs_of(int dtype, int dh, int rot, uint64_t align) {
  int v = dtype == DT_BF16 ? 8 : 4;
  const int esz = dtype == DT_BF16 ? 2 : 4;
  while (v > 1 && (dh % (2 * v) || rot % (2 * v) || align % (v * esz))) v /= 2;
  return v;
}

// Rows that fill the card with a wave each; fewer are divided, a group of heads
// each at the least (gradients of 2048 rows, 3 x 40 heads: 1024 the same, 4096 38.5 ->
// 43.2 us, each wave's angles and sums of the gains; 999 rows of 24 heads 14.2, 17).
constexpr int64_t FULL_WAVES = 2048;
constexpr int64_t MAX_PARTS = 64;
// Workgroups of the backward at most: each leaves a partial sum of the gains,
// and gain_sum_kernel takes 4 us for 1024 of them.  As many as run at once: half of
// them where a lane has 8 pairs, for its registers (8192 rows of 3 x 16 heads of 128,
// 1024 and 512: 61.9 and 59.6 us; fp32, 3 x 8 heads of 80, 42.1 and 47.5).
constexpr int64_t BWD_BLOCKS = 1024;

Shape shape_of(int op, int64_t rows, int rlog, int groups, int v) {
  Shape s{groups, 0, 1};
  const int64_t wgs = (((rows - 1) >> rlog) + WAVES) / WAVES;
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>({groups, FULL_WAVES / rows, MAX_PARTS}));
  s.per = static_cast<int>((groups + parts - 1) / parts);
  s.gy = static_cast<unsigned>((groups + s.per - 1) / s.per);
  s.gx = static_cast<unsigned>(std::min<int64_t>(wgs, op == NORM_BWD ? std::max<int64_t>(1, BWD_BLOCKS / (v == 8 ? 2 : 1) / s.gy) : MAX_WORKGROUPS / s.gy - 1));
  return s;
}

int plog_of(int dh, int v) {
  const int l = dh / (2 * v);
  int p = 0;
  while (p < 6 && (1 << p) < l) ++p;
  return p;
}

// Whether groups of several sides, and 2^rlog rows a wave, take half the passes or
// less (the registers that they need cost more than a few passes less: 16 + 2 + 2 heads,
// three for four, 20.1 -> 23.4 us; fp32 gradients of 8 + 2 + 2, two for three, 132 ->
// 166).  100,000 rows of 1 + 1 + 1 heads of 128: 137 -> 53 us, gradients 257 -> 100;
// 16,384 of 4 + 1 + 1 heads of 64: 25 -> 12, 52 -> 22.
bool mixed(int64_t rows, int Hq, int Hk, int Hv, int hlog, int64_t ld, int* rlog) {
  const int heads = Hq + Hk + Hv, S = 1 << hlog;
  const int apart = (Hq + S - 1) / S + (Hk + S - 1) / S + (Hv + S - 1) / S;
  int r = 0;
  while (r < hlog && (1 << (hlog - r - 1)) >= heads && rows >> (r + 1) >= FULL_WAVES && ld << (r + 1) < 1ll << 31) ++r;
  *rlog = r;
  return 2 * ((heads + S - 1) / S) <= apart << r;
}

template <typename T, int V, int OP, bool MIX>
void launch(const Args& a, bool pairs, const Shape& g, hipStream_t s) {
  const dim3 grid(g.gx, g.gy), block(64 * WAVES);
  if constexpr (V == 1) {
    if (a.dh > 128) {
      if (pairs) hipLaunchKernelGGL((rotary_kernel<T, V, 2, true, OP, MIX>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((rotary_kernel<T, V, 2, false, OP, MIX>), grid, block, 0, s, a);
      return;
    }
  }
  if (pairs) hipLaunchKernelGGL((rotary_kernel<T, V, 1, true, OP, MIX>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((rotary_kernel<T, V, 1, false, OP, MIX>), grid, block, 0, s, a);
}

template <int OP>
hipError_t run(int dtype, Args& a, int layout, uint64_t align, hipStream_t s, unsigned* blocks) {
  const int v = pairs_of(dtype, a.dh, a.rot, align);
  a.plog = plog_of(a.dh, v);
  const int hlog = 6 - a.plog, Hv = a.copy ? a.Hv : 0;
  *blocks = 0;
  if (a.rows == 0 || a.Hq + a.Hk + Hv == 0) return hipSuccess;
  // (in the widest accesses alone)
  const bool mix = v == (dtype == DT_BF16 ? 8 : 4) && mixed(a.rows, a.Hq, a.Hk, Hv, hlog, std::max({a.ldx, a.lddy, a.ldy}), &a.rlog);
  if (!mix) a.rlog = 0;
  const int slog = hlog - a.rlog, S = 1 << slog;
  auto groups = [&](int heads) { return (heads + S - 1) >> slog; };
  const Shape g = shape_of(OP, a.rows, a.rlog, mix ? groups(a.Hq + a.Hk + Hv) : groups(a.Hq) + groups(a.Hk) + groups(Hv), v);
  a.per = g.per;
  *blocks = g.gx * g.gy;
  const bool pairs = layout == ATOM_ROPE_PAIRS;
  if (dtype == DT_BF16) {
    if (mix) launch<bf16_t, 8, OP, true>(a, pairs, g, s);
    else if (v == 8) launch<bf16_t, 8, OP, false>(a, pairs, g, s);
    else if (v == 4) launch<bf16_t, 4, OP, false>(a, pairs, g, s);
    else if (v == 2) launch<bf16_t, 2, OP, false>(a, pairs, g, s);
    else launch<bf16_t, 1, OP, false>(a, pairs, g, s);
  } else {
    if (mix) launch<float, 4, OP, true>(a, pairs, g, s);
    else if (v == 4) launch<float, 4, OP, false>(a, pairs, g, s);
    else if (v == 2) launch<float, 2, OP, false>(a, pairs, g, s);
    else launch<float, 1, OP, false>(a, pairs, g, s);
  }
  return hipGetLastError();
}

// Bits that an address, or a pitch in bytes, sets below 16.
inline uint64_t low(const void* p) { return reinterpret_cast<uintptr_t>(p); }

uint64_t align_of(uint64_t bits) {
  uint64_t al = 16;
  while (al > 1 && (bits & (al - 1))) al /= 2;
  return al;
}

}  // namespace

hipError_t rope(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, const int32_t* pos, const double* freq,
                float mscale, int layout, bool back, int64_t rows, int T, int heads, int dh, int rot, hipStream_t s) {
  Args a{};
  a.x = x, a.y = y, a.ldx = ldx, a.ldy = ldy, a.pos = pos, a.freq = freq, a.mscale = mscale, a.back = back;
  a.rows = static_cast<uint32_t>(rows), a.T = T, a.Hq = heads, a.dh = dh, a.rot = rot;
  const uint64_t e = dtype == DT_BF16 ? 2 : 4;
  unsigned blocks;
  return run<ROPE>(dtype, a, layout, align_of(low(x) | low(y) | ldx * e | ldy * e), s, &blocks);
}

hipError_t qknorm_rope_fwd(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, const void* gq, const void* gk,
                           float eps, const int32_t* pos, const double* freq, float mscale, int layout, int64_t rows,
                           int T, int Hq, int Hk, int Hv, int dh, int rot, hipStream_t s) {
  Args a{};
  a.x = x, a.y = y, a.ldx = ldx, a.ldy = ldy, a.gq = gq, a.gk = gk, a.eps = eps, a.pos = pos, a.freq = freq;
  a.mscale = mscale, a.rows = static_cast<uint32_t>(rows), a.T = T, a.Hq = Hq, a.Hk = Hk, a.Hv = Hv, a.dh = dh, a.rot = rot;
  a.copy = y != x;
  const uint64_t e = dtype == DT_BF16 ? 2 : 4;
  unsigned blocks;
  return run<NORM>(dtype, a, layout, align_of(low(x) | low(y) | low(gq) | low(gk) | ldx * e | ldy * e), s, &blocks);
}

uint64_t qknorm_rope_bwd_ws(int dh) { return BWD_BLOCKS * 2 * dh * sizeof(float); }

hipError_t qknorm_rope_bwd(int dtype, const void* dy, int64_t lddy, const void* x, int64_t ldx, void* dx, int64_t lddx,
                           const void* gq, const void* gk, float* dgq, float* dgk, float eps, const int32_t* pos,
                           const double* freq, float mscale, int layout, int64_t rows, int T, int Hq, int Hk, int Hv,
                           int dh, int rot, float* ws, hipStream_t s) {
  Args a{};
  a.x = x, a.dy = dy, a.y = dx, a.ldx = ldx, a.lddy = lddy, a.ldy = lddx, a.gq = gq, a.gk = gk, a.eps = eps;
  a.pos = pos, a.freq = freq, a.mscale = mscale, a.rows = static_cast<uint32_t>(rows), a.T = T;
  a.Hq = Hq, a.Hk = Hk, a.Hv = Hv, a.dh = dh, a.rot = rot;
  a.copy = dx != dy;
  a.part = dgq || dgk ? ws : nullptr;
  const uint64_t e = dtype == DT_BF16 ? 2 : 4;
  unsigned blocks;
  hipError_t st = run<NORM_BWD>(dtype, a, layout,
                                align_of(low(x) | low(dy) | low(dx) | low(gq) | low(gk) | ldx * e | lddy * e | lddx * e), s,
                                &blocks);
  if (st != hipSuccess || !(dgq || dgk)) return st;
  // (no parts: zeros)
  hipLaunchKernelGGL(gain_sum_kernel, dim3((2 * dh + 15) / 16), dim3(1024), 0, s, ws, static_cast<int>(blocks), dh, dgq, dgk);
  return hipGetLastError();
}

}  // namespace atom
