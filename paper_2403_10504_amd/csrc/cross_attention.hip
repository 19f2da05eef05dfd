// Cross attention (atom_k_cross_attn_fwd, _bwd): queries of one sequence on the
// keys and values of another, of another length, heads of keys shared by groups
// of query heads.  bf16 kernels, and the launchers of both types.
//
//   z = scale q k^T;  lse = log sum exp z;  o = exp(z - lse) v
//   D = sum do o;  p = exp(z - lse);  ds = p (do v^T - D)
//   dv = p^T do;  dq = scale ds k;  dk = scale ds^T q
//
// The tiles are those of the causal attention (attention_kernels.h): a wave owns
// 16 rows or two times 16, key (or query) tiles of 64 rows go straight from
// memory to LDS, two stages; the scores stay in registers, S^T = K Q^T feeding
// the second product's operand; every output has one owner, so no atomics.  p and
// ds are rounded to bf16 for the second products (the operands' type: half a step
// of 2^-8 in each term, in random directions); sums and statistics are fp32.
//
// What bounds it: long sequences the vector unit and the matrix cores, which
// share a SIMD's issue slots (2 x 2048 queries, 4096 keys, 32 heads of 128: 259 us,
// 1.06 PFLOP/s, matrix cores busy 46 %; a library product here 1.43); short ones
// the bytes of q and o and the start of a workgroup (8 x 2048 queries on 48 to 500
// keys, 12 heads of 64: 31 us, of which 15 remain with 64 keys); single tokens the
// keys' bytes (8 x 1 on 261 to 2048 keys, 40 heads of 128: 51 us, 4.5 TB/s).
#include "cross_attention.h"

#include "../../include/atom.h"
#include "../../include/atom_kernels.h"

namespace atom {
namespace cross {

using namespace attn;

// Fragment of packed row p of a head group (zeros behind the last).
template <int DH>
ATOM_DEV void frag_row(Frag<bf16_t>& f, const CrossArgs& a, const bf16_t* base, const Seq& s, int hk, int p, int P,
                       int64_t ld, int col) {
  if (p < P) frag_load(f, base + at<DH>(a, s, hk, p, ld) + col);
  else frag_zero(f);
}

// Makes the compiler wait for a fragment's load here: it places its waits at the
// first use, and one inside a tile loop, which it cannot count past the direct
// loads that it does not see, is a wait for all of them in every tile.
ATOM_DEV void settle(Frag<bf16_t>& f) { asm volatile("" : "+v"(f.v.x), "+v"(f.v.y), "+v"(f.v.z), "+v"(f.v.w)); }

// Direct loads by a tile's base (scalar) and the lane's 32-bit offset in it
// (leading dimensions below 2^24: 64 rows stay within 2^32 bytes).
ATOM_DEV void lds_dma16_at(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0"
               :
               : "s"(base), "v"(off), "s"(lds)
               : "memory", "m0");
}

// The tiles of a range.
struct Range {
  int t0, t1;
};
ATOM_DEV Range range_of(int n_rows, int splits, int s) {
  const int n = (n_rows + BT - 1) / BT, per = (n + splits - 1) / splits;
  return Range{min(s * per, n), min(s * per + per, n)};
}

// Every wave is done with the stages in LDS.
ATOM_DEV void stages_done() {
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  asm volatile("s_barrier" ::: "memory");
}
// A wave's results go out through LDS (the stages' place), N rows of DH, so that a
// store covers whole rows instead of 32 bytes of each (one tile of keys 25.5 -> 22.6
// us; gradients of 4 x 64 x 1500, 32 heads of 128, 108 -> 96, of 2 x 512 x 16000, 8 heads,
// 291 -> 281).
template <int DH, int N>
struct Rows {
  static constexpr int RB = DH * 2, CPR = DH / 8;  // bytes and chunks of 16 bytes in a row
  uint8_t* mine;
  // columns 16 c + 4 lg + 0..3 of a row
  ATOM_DEV void put(int row, int c, int lg, float (&v)[4]) const {
    const int chunk = (2 * c + (lg >> 1)) ^ (row & (CPR - 1));
    store_row4<bf16_t>(reinterpret_cast<bf16_t*>(mine + row * RB + chunk * 16 + 8 * (lg & 1)), v);
  }
  // to(row, on): where a row goes, and whether it does
  template <typename TO>
  ATOM_DEV void store(int lane, TO to) const {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < N * CPR / 64; ++i) {
      const int row = i * (64 / CPR) + lane / CPR, chunk = lane % CPR;
      const uint4 v = *reinterpret_cast<const uint4*>(mine + row * RB + (chunk ^ (row & (CPR - 1))) * 16);
      bool on;
      bf16_t* p = to(row, on);
      if (on) *reinterpret_cast<uint4*>(p + chunk * 8) = v;
    }
  }
};

// ------------------------------------------------------------------ forward
// A tile's scores are computed one tile ahead: the matrix instructions of
// S(t+1) = K Q^T stand between the exponentials of P(t), which need nothing of
// them, so that both units work in one wave.  K is staged one tile ahead of V.
// (2 x 2048 x 4096, 32 heads of 128: 16 rows a wave, one tile after the other 311
// us, 32 rows 308 to 310; ahead 275 in 256-row workgroups, 289 in 128-row ones, 360
// with 16 rows a wave; without branches between the score and the second product 260
// and 275.  Orders asked for by scheduling groups: 266 to 270; two score tiles' sums
// side by side, 3 to 6 fragments of V ahead: within 2 us; the two halves of a
// workgroup in turns, one in its products while the other has its exponentials, two
// barriers a tile: 262; 64 rows a wave at one wave a SIMD spill: 349.)
template <int DH, int GR, int NW, bool SPLIT>
__global__ void __launch_bounds__(64 * NW, 2) cross_fwd_kernel(const CrossArgs a) {
  constexpr int NT = 64 * NW;
  using F = FwdDL<DH, NT>;
  constexpr int NS = DH / 32, NCT = DH / 16, BQ = NW * 16 * GR, RB = DH * 2;
  constexpr int ROWS = NT / F::CPR;  // rows of a tile that the workgroup loads at once
  static_assert(ROWS % 16 == 0, "swizzles repeat from load to load");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * F::TILE];  // K, K, V, V

  const int BH = a.B * a.Hk;
  const int item = item_of(a.n_x * BH * a.splits, blockIdx.x);
  if (item < 0) return;
  const int x = item % a.n_x, split = SPLIT ? item / a.n_x % a.splits : 0, bh = item / (a.n_x * a.splits);
  const int b = bh % a.B, hk = bh / a.B;  // (see item_of)
  const Seq qs = seq(a.q_start, a.q_len, a.Tq, a.q_rows, b), ks = seq(a.k_start, a.k_len, a.Tk, a.k_rows, b);
  const int P = qs.n * a.G, n_keys = ks.n;
  const int q0 = x * BQ;
  if (q0 >= P && (SPLIT || a.q_start)) return;

  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int qw = q0 + w * 16 * GR;
  const float sc = a.scale * LOG2E;
  const bf16_t* qb = static_cast<const bf16_t*>(a.q);
  const bf16_t* kb = static_cast<const bf16_t*>(a.k) + ks.row0 * a.ldk + hk * DH;
  const bf16_t* vb = static_cast<const bf16_t*>(a.v) + ks.row0 * a.ldv + hk * DH;

  // Row and chunk of a thread's loads; the last, partial tile reads its last
  // key again (whose scores are masked).
  const int lrow = tid / F::CPR, slot = tid % F::CPR;
  const uint32_t k_col = (slot ^ F::kswz(lrow)) * 16, v_col = (slot ^ F::vswz(lrow)) * 16;
  auto load_tile = [&](const bf16_t* base, int64_t ld, uint32_t col, int at_lds, int j0) {
    const bf16_t* tile = base + j0 * ld;
    const uint32_t pitch = static_cast<uint32_t>(ld) * 2, dst = lds_offset(lds + at_lds) + w * 1024;
    const bool whole = j0 + BT <= n_keys;
#pragma unroll
    for (int q = 0; q < F::LPT; ++q) {
      const int row = whole ? lrow + q * ROWS : min(lrow + q * ROWS, n_keys - 1 - j0);
      lds_dma16_at(tile, row * pitch + col, __builtin_amdgcn_readfirstlane(dst + q * NT * 16));
    }
  };
  auto load_k = [&](int kt) { load_tile(kb, a.ldk, k_col, (kt & 1) * F::TILE, kt * BT); };
  auto load_v = [&](int kt) { load_tile(vb, a.ldv, v_col, (2 + (kt & 1)) * F::TILE, kt * BT); };
  // every load has landed, for every wave, and every wave is done with the stages before
  auto fence = [&] {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    asm volatile("s_barrier" ::: "memory");
  };

  const Range rg = q0 < P ? range_of(n_keys, a.splits, split) : Range{0, 0};
  if (rg.t0 < rg.t1) {
    load_k(rg.t0);
    load_v(rg.t0);
  }

  Frag<bf16_t> qf[GR][NS];
#pragma unroll
  for (int g = 0; g < GR; ++g)
#pragma unroll
    for (int s = 0; s < NS; ++s) frag_row<DH>(qf[g][s], a, qb, qs, hk, qw + g * 16 + lr, P, a.ldq, 32 * s + 8 * lg);

  f32x4_t acc_o[GR][NCT];
  float m_i[GR], l_i[GR], mloc[GR];
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    m_i[g] = NO_MAX;
    l_i[g] = 0.f;
#pragma unroll
    for (int c = 0; c < NCT; ++c) acc_o[g][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  auto kfrag = [&](Frag<bf16_t>& f, const uint8_t* st, int jt, int s) {
    const int row = jt * 16 + lr;
    f.v = *reinterpret_cast<const uint4*>(st + row * RB + ((4 * s + lg) ^ F::kswz(row)) * 16);
  };
  auto vfrag = [&](Frag<bf16_t>& f, const uint8_t* st, int s2, int c) {
    // keys 32 s2 + 4 lg + 0..3 and 32 s2 + 16 + 4 lg + 0..3, the order of the
    // P fragment built from two 16-key tiles
    const int chunk = 2 * c + ((lr & 3) >> 1);
    const int r0 = 32 * s2 + 4 * lg + (lr >> 2), r1 = r0 + 16;
    const uint2 lo = ds_read_tr8(st + r0 * RB + (chunk ^ F::vswz(r0)) * 16 + 8 * (lr & 1));
    const uint2 hi = ds_read_tr8(st + r1 * RB + (chunk ^ F::vswz(r1)) * 16 + 8 * (lr & 1));
    f.v = make_uint4(lo.x, lo.y, hi.x, hi.y);
  };
  // z = raw scores of tile kt, `between` standing between the matrix
  // instructions of its four parts
  auto scores = [&](float (&z)[GR][4][4], int kt, auto between) {
    const uint8_t* st = lds + (kt & 1) * F::TILE;
    Frag<bf16_t> kf[2][NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) kfrag(kf[0][s], st, 0, s);
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      if (jt + 1 < 4) {
#pragma unroll
        for (int s = 0; s < NS; ++s) kfrag(kf[(jt + 1) & 1][s], st, jt + 1, s);
      }
      f32x4_t c[GR];
#pragma unroll
      for (int g = 0; g < GR; ++g) c[g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int g = 0; g < GR; ++g) mfma16(c[g], kf[jt & 1][s], qf[g][s]);
      between(jt);
#pragma unroll
      for (int g = 0; g < GR; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) z[g][jt][r] = c[g][r];
    }
  };
  // a tile's scores behind the last key: -infinity
  auto mask = [&](float (&z)[GR][4][4], int kt) {
#pragma unroll
    for (int jt = 0; jt < 4; ++jt)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int g = 0; g < GR; ++g)
          z[g][jt][r] = kt * BT + jt * 16 + 4 * lg + r < n_keys ? z[g][jt][r] : -INFINITY;
  };
  auto maxima = [&](const float (&z)[GR][4][4]) {
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      float m = -INFINITY;
#pragma unroll
      for (int jt = 0; jt < 4; ++jt)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, z[g][jt][r]);
      mloc[g] = m;
    }
  };
  // One tile: its exponentials and its part of O, and the scores of the next
  // (NEXT 0: none; 1: a whole one; 2: the last).  Without branches from the
  // first score on, so that the compiler's order is the one asked for.
  auto step = [&](auto NEXT_, float (&z)[GR][4][4], float (&next)[GR][4][4], int kt) {
    constexpr int NEXT = decltype(NEXT_)::value;
    // of a SIMD's waves the one that has exponentials to do goes first, so that they
    // come apart (cross_small 32.0 -> 30.9 us, cross_6.7b 261 -> 257)
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      const float mx = rows4_max(mloc[g]) * sc;
      // the reference is raised only where a score is beyond it by 2^8
      if (__builtin_amdgcn_ballot_w64(mx > m_i[g] + RESCALE_LOG2) != 0) {
        const float m_new = fmaxf(m_i[g], mx);
        const float alpha = ex2(m_i[g] - m_new);
        l_i[g] *= alpha;
        m_i[g] = m_new;
#pragma unroll
        for (int c = 0; c < NCT; ++c) acc_o[g][c] *= alpha;
      }
    }
    fence();
    if (NEXT && kt + 2 < rg.t1) load_k(kt + 2);
    if (NEXT) load_v(kt + 1);
    auto exps = [&](int jt) {
#pragma unroll
      for (int g = 0; g < GR; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          z[g][jt][r] = ex2(__builtin_fmaf(z[g][jt][r], sc, -m_i[g]));
          l_i[g] += z[g][jt][r];
        }
    };
    if constexpr (NEXT != 0) {
      scores(next, kt + 1, exps);
    } else {
#pragma unroll
      for (int jt = 0; jt < 4; ++jt) exps(jt);
    }
    __builtin_amdgcn_s_setprio(0);
    const uint8_t* vst = lds + (2 + (kt & 1)) * F::TILE;
    constexpr int AHEAD = 4;  // fragments of V in flight
    Frag<bf16_t> vf[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) vfrag(vf[n], vst, n / NCT, n % NCT);
    if constexpr (NEXT == 2) {
      if (kt * BT + 2 * BT > n_keys) mask(next, kt + 1);
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      Frag<bf16_t> pf[GR];
#pragma unroll
      for (int g = 0; g < GR; ++g) frag_from_pair(pf[g], z[g], s2);
#pragma unroll
      for (int c = 0; c < NCT; ++c) {
        const int n = s2 * NCT + c;
#pragma unroll
        for (int g = 0; g < GR; ++g) mfma16(acc_o[g][c], vf[n % AHEAD], pf[g]);
        if (n + AHEAD < 2 * NCT) vfrag(vf[n % AHEAD], vst, (n + AHEAD) / NCT, (n + AHEAD) % NCT);
      }
    }
    if constexpr (NEXT != 0) maxima(next);
  };
  if (rg.t0 < rg.t1) {
    float z0[GR][4][4], z1[GR][4][4];
    using None = std::integral_constant<int, 0>;
    using Whole = std::integral_constant<int, 1>;
    using Last = std::integral_constant<int, 2>;
    fence();
#pragma unroll
    for (int g = 0; g < GR; ++g)
#pragma unroll
      for (int s = 0; s < NS; ++s) settle(qf[g][s]);
    if (rg.t0 + 1 < rg.t1) load_k(rg.t0 + 1);
    scores(z0, rg.t0, [](int) {});
    if (rg.t0 * BT + BT > n_keys) mask(z0, rg.t0);
    maxima(z0);
    int kt = rg.t0;
    for (; kt + 3 < rg.t1; kt += 2) {
      step(Whole{}, z0, z1, kt);
      step(Whole{}, z1, z0, kt + 1);
    }
    // one to three tiles
    auto move = [&] {
#pragma unroll
      for (int g = 0; g < GR; ++g)
#pragma unroll
        for (int jt = 0; jt < 4; ++jt)
#pragma unroll
          for (int r = 0; r < 4; ++r) z0[g][jt][r] = z1[g][jt][r];
      ++kt;
    };
    if (kt + 2 < rg.t1) {
      step(Whole{}, z0, z1, kt);
      move();
    }
    if (kt + 1 < rg.t1) {
      step(Last{}, z0, z1, kt);
      move();
    }
    step(None{}, z0, z1, kt);
  }

  if constexpr (SPLIT) {
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      const int pi = qw + g * 16 + lr;
      const float l_tot = rows4_sum(l_i[g]);
      if (pi >= P) continue;
      const int64_t n = static_cast<int64_t>(a.Tq) * a.G, r = (static_cast<int64_t>(split) * BH + bh) * n + pi;
#pragma unroll
      for (int c = 0; c < NCT; ++c) {
        float v[4] = {acc_o[g][c][0], acc_o[g][c][1], acc_o[g][c][2], acc_o[g][c][3]};
        store_row4<float>(a.part + r * DH + c * 16 + 4 * lg, v);
      }
      if (lg == 0) a.ml[2 * r] = m_i[g], a.ml[2 * r + 1] = l_tot;
    }
    return;
  }
  constexpr int WROWS = 16 * GR;
  static_assert(NW * WROWS * RB <= 4 * F::TILE, "results in the stages' place");
  Rows<DH, WROWS> out{lds + w * WROWS * RB};
  fence();
  // padded queries of a padded batch get zeros (P up to Tq G)
  const int p_end = a.q_start ? P : a.Tq * a.G;
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    const int row = g * 16 + lr, pi = qw + row;
    const float l_tot = rows4_sum(l_i[g]);
    const bool none = l_tot == 0.f || pi >= P;  // no keys, or padding: zeros
    const float inv = 1.f / l_tot;
#pragma unroll
    for (int c = 0; c < NCT; ++c) {
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = none ? 0.f : acc_o[g][c][r] * inv;
      out.put(row, c, lg, v);
    }
    if (lg == 0 && a.lse && pi < p_end) {
      const Row rw = row_of(a, pi);
      a.lse[(qs.row0 + rw.t) * a.Hq + hk * a.G + rw.g] = none ? -INFINITY : (m_i[g] + log2f(l_tot)) * LN2;
    }
  }
  out.store(lane, [&](int row, bool& on) {
    on = qw + row < p_end;
    return static_cast<bf16_t*>(a.o) + (on ? at<DH>(a, qs, hk, qw + row, a.ldo) : 0);
  });
}

// ------------------------------------------------------------ backward: dQ
// Also D of every row, for a dK/dV kernel that reads it (a.dq null: D alone).
// 32 queries a wave in large problems, which halves the LDS reads of K and V (2 x
// 2048 x 1500, 32 heads of 128: 203 us with 16, 155 with 32: 0.98 PFLOP/s of its
// three products).
template <int DH, int GR, int NW>
ATOM_DEV void dq_body(uint8_t* lds, const CrossArgs& a, int item) {
  using F = FwdDL<DH>;
  constexpr int NS = DH / 32, NCT = DH / 16, BQ = NW * 16 * GR, NT = 64 * NW, RB = DH * 2;
  constexpr int LPT = F::TILE / (NT * 16), ROWS = NT / F::CPR;
  static_assert(ROWS % 16 == 0, "swizzles repeat from load to load");

  const int BH = a.B * a.Hk;
  const bool ranges = a.splits > 1;
  const int x = item % a.n_x, split = item / a.n_x % a.splits, bh = item / (a.n_x * a.splits);
  const int b = bh % a.B, hk = bh / a.B;  // (see item_of)
  const Seq qs = seq(a.q_start, a.q_len, a.Tq, a.q_rows, b), ks = seq(a.k_start, a.k_len, a.Tk, a.k_rows, b);
  const int P = qs.n * a.G, n_keys = ks.n;
  const int q0 = x * BQ;
  if (q0 >= P && (ranges || a.q_start)) return;
  const int64_t n_p = static_cast<int64_t>(a.Tq) * a.G;

  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int qw = q0 + w * 16 * GR;
  const float sc = a.scale * LOG2E;
  const bf16_t* kb = static_cast<const bf16_t*>(a.k) + ks.row0 * a.ldk + hk * DH;
  const bf16_t* vb = static_cast<const bf16_t*>(a.v) + ks.row0 * a.ldv + hk * DH;

  const int lrow = tid / F::CPR, slot = tid % F::CPR;
  const uint32_t k_col = (slot ^ dsw<DH>(lrow)) * 16, v_col = (slot ^ F::kswz(lrow)) * 16;
  auto load_tile = [&](int st, int j0) {
    const uint32_t dst = lds_offset(lds + st * F::STAGE) + w * 1024;
    const bf16_t *kt = kb + j0 * a.ldk, *vt = vb + j0 * a.ldv;
    const uint32_t kp = static_cast<uint32_t>(a.ldk) * 2, vp = static_cast<uint32_t>(a.ldv) * 2;
#pragma unroll
    for (int q = 0; q < LPT; ++q) {
      const uint32_t row = min(lrow + q * ROWS, n_keys - 1 - j0);
      lds_dma16_at(kt, row * kp + k_col, __builtin_amdgcn_readfirstlane(dst + q * NT * 16));
      lds_dma16_at(vt, row * vp + v_col, __builtin_amdgcn_readfirstlane(dst + F::TILE + q * NT * 16));
    }
  };
  const Range rg = q0 < P && a.dq ? range_of(n_keys, a.splits, split) : Range{0, 0};
  if (rg.t0 < rg.t1) load_tile(0, rg.t0 * BT);

  Frag<bf16_t> qf[GR][NS], of[GR][NS];
  float lse_i[GR], del_i[GR];
  f32x4_t acc[GR][NCT];
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    const int pi = qw + g * 16 + lr;
    lse_i[g] = INFINITY;
    if (pi < P) {
      const Row rw = row_of(a, pi);
      lse_i[g] = lse2_of(a.lse[(qs.row0 + rw.t) * a.Hq + hk * a.G + rw.g]);
    }
    Frag<bf16_t> f[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      frag_row<DH>(qf[g][s], a, static_cast<const bf16_t*>(a.q), qs, hk, pi, P, a.ldq, 32 * s + 8 * lg);
      frag_row<DH>(of[g][s], a, static_cast<const bf16_t*>(a.dout), qs, hk, pi, P, a.lddo, 32 * s + 8 * lg);
      frag_row<DH>(f[s], a, static_cast<const bf16_t*>(a.o), qs, hk, pi, P, a.ldo, 32 * s + 8 * lg);
    }
#pragma unroll
    for (int s = 0; s < NS; ++s) settle(qf[g][s]);
    del_i[g] = row_dot<NS>(f, of[g]);
    if (a.delta && lg == 0 && pi < P && split == 0) a.delta[bh * n_p + pi] = del_i[g];
#pragma unroll
    for (int c = 0; c < NCT; ++c) acc[g][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
#pragma unroll
  for (int g = 0; g < GR; ++g) asm volatile("" : "+v"(lse_i[g]), "+v"(del_i[g]));
  if (!a.dq) return;
  auto rowfrag = [&](Frag<bf16_t>& f, const uint8_t* st, int jt, int s, bool dual) {
    const int row = jt * 16 + lr, chunk = 4 * s + lg;
    f.v = *reinterpret_cast<const uint4*>(st + row * RB + (chunk ^ (dual ? dsw<DH>(row) : F::kswz(row))) * 16);
  };
  auto trfrag = [&](Frag<bf16_t>& f, const uint8_t* st, int s2, int c) {
    const int chunk = 2 * c + ((lr & 3) >> 1);
    const int r0 = 32 * s2 + 4 * lg + (lr >> 2), r1 = r0 + 16;
    const uint2 lo = ds_read_tr8(st + r0 * RB + (chunk ^ dsw<DH>(r0)) * 16 + 8 * (lr & 1));
    const uint2 hi = ds_read_tr8(st + r1 * RB + (chunk ^ dsw<DH>(r1)) * 16 + 8 * (lr & 1));
    f.v = make_uint4(lo.x, lo.y, hi.x, hi.y);
  };
  for (int kt = rg.t0; kt < rg.t1; ++kt) {
    const int cur = (kt - rg.t0) & 1;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    asm volatile("s_barrier" ::: "memory");
    if (kt + 1 < rg.t1) load_tile(cur ^ 1, (kt + 1) * BT);
    if (qw >= P) continue;
    // A loop of one trip, for the compiler: without it the same code takes more
    // registers (dQ of heads of 128, 32 queries a wave: 63 spilled in place of none,
    // 2 x 2048 x 1500, 32 heads, both gradients 366 -> 578 us).
#pragma unroll 1
    for (int once = 0; once < 1; ++once) {
      const int j0 = kt * BT;
      const uint8_t* kst = lds + cur * F::STAGE;
      const uint8_t* vst = kst + F::TILE;
      float ds[GR][4][4];
      auto score_tile = [&](auto MASK_) {
        constexpr bool MASK = decltype(MASK_)::value;
        Frag<bf16_t> kf[2][NS], vf[2][NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          rowfrag(kf[0][s], kst, 0, s, true);
          rowfrag(vf[0][s], vst, 0, s, false);
        }
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) {
          if (jt + 1 < 4) {
#pragma unroll
            for (int s = 0; s < NS; ++s) {
              rowfrag(kf[(jt + 1) & 1][s], kst, jt + 1, s, true);
              rowfrag(vf[(jt + 1) & 1][s], vst, jt + 1, s, false);
            }
          }
          f32x4_t sa[GR], dp[GR];
#pragma unroll
          for (int g = 0; g < GR; ++g) sa[g] = dp[g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int g = 0; g < GR; ++g) {
              mfma16(sa[g], kf[jt & 1][s], qf[g][s]);  // S^T[j][i]: lane holds one query, keys 4lg + r
              mfma16(dp[g], vf[jt & 1][s], of[g][s]);  // dP^T[j][i]
            }
#pragma unroll
          for (int g = 0; g < GR; ++g)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float pv = ex2(__builtin_fmaf(sa[g][r], sc, -lse_i[g]));
              float d = pv * (dp[g][r] - del_i[g]);
              if constexpr (MASK) d = j0 + jt * 16 + 4 * lg + r < n_keys ? d : 0.f;
              ds[g][jt][r] = d;
            }
        }
      };
      if (j0 + BT > n_keys) score_tile(std::true_type{});
      else score_tile(std::false_type{});
      constexpr int AHEAD = 2;
      Frag<bf16_t> kt2[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) trfrag(kt2[n], kst, n / NCT, n % NCT);
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        Frag<bf16_t> dsf[GR];
#pragma unroll
        for (int g = 0; g < GR; ++g) frag_from_pair(dsf[g], ds[g], s2);
#pragma unroll
        for (int c = 0; c < NCT; ++c) {
          const int n = s2 * NCT + c;
#pragma unroll
          for (int g = 0; g < GR; ++g) mfma16(acc[g][c], kt2[n % AHEAD], dsf[g]);  // dQ^T[c][i]
          if (n + AHEAD < 2 * NCT) trfrag(kt2[n % AHEAD], kst, (n + AHEAD) / NCT, (n + AHEAD) % NCT);
        }
      }
    }
  }

  Rows<DH, 16 * GR> out{lds + w * 16 * GR * RB};
  static_assert(NW * 16 * GR * RB <= 2 * F::STAGE, "results in the stages' place");
  if (!ranges) stages_done();
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    const int pi = qw + g * 16 + lr;
    if (ranges) {
      if (pi >= P) continue;
      float* row = a.part + ((static_cast<int64_t>(split) * BH + bh) * n_p + pi) * DH;
#pragma unroll
      for (int c = 0; c < NCT; ++c) {
        float v[4] = {acc[g][c][0], acc[g][c][1], acc[g][c][2], acc[g][c][3]};
        store_row4<float>(row + c * 16 + 4 * lg, v);
      }
      continue;
    }
#pragma unroll
    for (int c = 0; c < NCT; ++c) {
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = pi < P ? acc[g][c][r] * a.scale : 0.f;  // (padding: zeros)
      out.put(g * 16 + lr, c, lg, v);
    }
  }
  if (ranges) return;
  const int64_t p_end = a.q_start ? P : n_p;
  out.store(lane, [&](int row, bool& on) {
    on = qw + row < p_end;
    return static_cast<bf16_t*>(a.dq) + (on ? at<DH>(a, qs, hk, qw + row, a.lddq) : 0);
  });
}

// -------------------------------------------------------- backward: dK, dV
// OWN_D: D of the range's queries is computed here, from O and dO, into d_own
// (LDS); otherwise it is read from a.delta.
// Two waves a SIMD, which the accumulators of dK and dV and the fragments of K and V
// leave room for, do not hide all of the LDS reads and exponentials (2 x 2048 x 1500,
// 32 heads of 128: 217 us, 0.93 PFLOP/s of its four products, matrix cores busy 40 %,
// LDS 46 %).  Slower there: 32 keys a wave at one wave a SIMD (250), row fragments
// of two steps held (233), the second products beside the next step's scores (235),
// workgroups of four waves (246), three or four fragments ahead (224).
template <int DH, int W, int SUB, bool OWN_D>
ATOM_DEV void dkdv_body(uint8_t* lds, float* d_own, const CrossArgs& a, int item) {
  using F = FwdDL<DH>;
  constexpr int NS = DH / 32, NCT = DH / 16, NT = 64 * W, RB = DH * 2, BKEYS = 16 * W;
  constexpr int LPT = F::TILE / (NT * 16), ROWS = NT / F::CPR;
  static_assert(ROWS % 16 == 0, "swizzles repeat from load to load");
  constexpr int STAGE = dkdv_stage<DH>();

  const int BH = a.B * a.Hk;
  const bool ranges = a.k_splits > 1;
  const int x = item % a.k_x, split = item / a.k_x % a.k_splits, bh = item / (a.k_x * a.k_splits);
  const int b = bh % a.B, hk = bh / a.B;  // (see item_of)
  const Seq qs = seq(a.q_start, a.q_len, a.Tq, a.q_rows, b), ks = seq(a.k_start, a.k_len, a.Tk, a.k_rows, b);
  const int P = qs.n * a.G, n_keys = ks.n;
  const int k0 = x * BKEYS;
  if (k0 >= n_keys && (ranges || a.k_start)) return;
  const int64_t n_p = static_cast<int64_t>(a.Tq) * a.G;

  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int kw = k0 + w * 16, kj = kw + lr;
  const float sc = a.scale * LOG2E;
  const bf16_t* qb = static_cast<const bf16_t*>(a.q);
  const bf16_t* ob = static_cast<const bf16_t*>(a.dout);
  const bf16_t* kb = static_cast<const bf16_t*>(a.k) + ks.row0 * a.ldk + hk * DH;
  const bf16_t* vb = static_cast<const bf16_t*>(a.v) + ks.row0 * a.ldv + hk * DH;

  Frag<bf16_t> kf[NS], vf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    frag_global(kf[s], kb, a.ldk, kj, n_keys, 32 * s + 8 * lg);
    frag_global(vf[s], vb, a.ldv, kj, n_keys, 32 * s + 8 * lg);
  }
  f32x4_t acc_dk[NCT], acc_dv[NCT];
#pragma unroll
  for (int c = 0; c < NCT; ++c) {
    acc_dk[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    acc_dv[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  const int lrow = tid / F::CPR;
  const uint32_t col = ((tid % F::CPR) ^ dsw<DH>(lrow)) * 16;
  auto load_tile = [&](int st, int i0) {
    const uint32_t dst = lds_offset(lds + st * STAGE) + w * 1024;
    const int t0 = row_of(a, i0).t;  // the tile's first token: its rows are less than 2^32 bytes on
    const bf16_t *qt = qb + (qs.row0 + t0) * a.ldq, *ot = ob + (qs.row0 + t0) * a.lddo;
#pragma unroll
    for (int q = 0; q < LPT; ++q) {
      const Row rw = row_of(a, min(i0 + lrow + q * ROWS, P - 1));
      const uint32_t c = static_cast<uint32_t>(hk * a.G + rw.g) * (DH * 2) + col, t = rw.t - t0;
      lds_dma16_at(qt, t * (static_cast<uint32_t>(a.ldq) * 2) + c, __builtin_amdgcn_readfirstlane(dst + q * NT * 16));
      lds_dma16_at(ot, t * (static_cast<uint32_t>(a.lddo) * 2) + c, __builtin_amdgcn_readfirstlane(dst + F::TILE + q * NT * 16));
    }
  };
  // LSE and D of a stage's rows go through registers; rows past the end get
  // LSE = +inf, so their P is 0
  float pre_lse = 0.f, pre_del = 0.f;
  auto read_rows = [&](int i0) {
    if (tid < SUB * BT) {
      const int i = i0 + tid;
      pre_lse = INFINITY;
      pre_del = 0.f;
      if (i < P) {
        const Row rw = row_of(a, i);
        pre_lse = lse2_of(a.lse[(qs.row0 + rw.t) * a.Hq + hk * a.G + rw.g]);
        if constexpr (!OWN_D) pre_del = a.delta[bh * n_p + i];
      }
    }
  };
  auto store_rows = [&](int st) {
    if (tid < SUB * BT) {
      float* rows = reinterpret_cast<float*>(lds + (st * SUB + tid / BT) * STAGE + 2 * F::TILE);
      rows[tid % BT] = pre_lse;
      if constexpr (!OWN_D) rows[BT + tid % BT] = pre_del;
    }
  };
  auto rowfrag = [&](Frag<bf16_t>& f, const uint8_t* st, int it, int s) {
    const int row = it * 16 + lr, chunk = 4 * s + lg;
    f.v = *reinterpret_cast<const uint4*>(st + row * RB + (chunk ^ dsw<DH>(row)) * 16);
  };
  auto trfrag = [&](Frag<bf16_t>& f, const uint8_t* st, int s2, int c) {
    const int chunk = 2 * c + ((lr & 3) >> 1);
    const int r0 = 32 * s2 + 4 * lg + (lr >> 2), r1 = r0 + 16;
    const uint2 lo = ds_read_tr8(st + r0 * RB + (chunk ^ dsw<DH>(r0)) * 16 + 8 * (lr & 1));
    const uint2 hi = ds_read_tr8(st + r1 * RB + (chunk ^ dsw<DH>(r1)) * 16 + 8 * (lr & 1));
    f.v = make_uint4(lo.x, lo.y, hi.x, hi.y);
  };

  const Range rg = k0 < n_keys ? range_of(P, a.k_splits, split) : Range{0, 0};
  auto load_stage = [&](int st, int qt) {
#pragma unroll
    for (int u = 0; u < SUB; ++u)
      if (qt + u < rg.t1) load_tile(st * SUB + u, (qt + u) * BT);
  };
  if (rg.t0 < rg.t1) {
    load_stage(0, rg.t0);
    read_rows(rg.t0 * BT);
    store_rows(0);
  }
  if constexpr (OWN_D) {
    // 16 queries a wave and step, FLY steps' loads in flight; rows past the end
    // are zeros.  The loop's first barrier makes d_own visible.
    constexpr int FLY = 2;
    for (int r0 = rg.t0 * BT; r0 < rg.t1 * BT; r0 += 16 * W * FLY) {
      Frag<bf16_t> fo[FLY][NS], fd[FLY][NS];
#pragma unroll
      for (int f = 0; f < FLY; ++f)
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const int r = r0 + 16 * (f * W + w) + lr;
          frag_row<DH>(fo[f][s], a, static_cast<const bf16_t*>(a.o), qs, hk, r, P, a.ldo, 32 * s + 8 * lg);
          frag_row<DH>(fd[f][s], a, ob, qs, hk, r, P, a.lddo, 32 * s + 8 * lg);
        }
#pragma unroll
      for (int f = 0; f < FLY; ++f) {
        const int r = r0 + 16 * (f * W + w) + lr;
        const float v = row_dot<NS>(fo[f], fd[f]);
        if (lg == 0 && r < rg.t1 * BT) d_own[r - rg.t0 * BT] = v;
      }
    }
  }
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    settle(kf[s]);
    settle(vf[s]);
  }
  for (int qs0 = rg.t0; qs0 < rg.t1; qs0 += SUB) {
    const int cur = ((qs0 - rg.t0) / SUB) & 1;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    asm volatile("s_barrier" ::: "memory");
    const bool more = qs0 + SUB < rg.t1;
    if (more) {
      load_stage(cur ^ 1, qs0 + SUB);
      read_rows((qs0 + SUB) * BT);
    }
#pragma unroll 1
    for (int u = 0; u < SUB; ++u) {
      if (qs0 + u >= rg.t1 || kw >= n_keys) break;
      const uint8_t* qst = lds + (cur * SUB + u) * STAGE;
      const uint8_t* ost = qst + F::TILE;
      const float* lse_s = reinterpret_cast<const float*>(qst + 2 * F::TILE);
      const float* del_s = OWN_D ? d_own + (qs0 + u - rg.t0) * BT : lse_s + BT;
      float p[4][4], ds[4][4];
      // Keys past the end need no mask: their columns are never stored, and
      // their fragments are zeros.  Each step's LDS reads stand before the
      // exponentials of the step before, and stay there (hoisted, they spill).
      Frag<bf16_t> qf[NS], of[NS];
      auto read = [&](int it) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          rowfrag(qf[s], qst, it, s);
          rowfrag(of[s], ost, it, s);
        }
      };
      constexpr int AHEAD = 2;
      Frag<bf16_t> ot2[AHEAD], qt2[AHEAD];
      __builtin_amdgcn_s_setprio(1);  // (as in the forward: 219 -> 217 us)
      read(0);
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        f32x4_t sa = f32x4_t{0.f, 0.f, 0.f, 0.f}, dp = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          mfma16(sa, qf[s], kf[s]);  // S[i][j]: lane holds key kj, queries 4lg + r
          mfma16(dp, of[s], vf[s]);  // dP[i][j]
        }
        if (it + 1 < 4) {
          read(it + 1);
        } else {
#pragma unroll
          for (int n = 0; n < AHEAD; ++n) {
            trfrag(ot2[n], ost, 0, n);
            trfrag(qt2[n], qst, 0, n);
          }
        }
        __builtin_amdgcn_sched_barrier(0x000A);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int il = it * 16 + 4 * lg + r;
          p[it][r] = ex2(__builtin_fmaf(sa[r], sc, -lse_s[il]));
          ds[it][r] = p[it][r] * (dp[r] - del_s[il]);
        }
      }
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        Frag<bf16_t> pf, dsf;
        frag_from_pair(pf, p, s2);
        frag_from_pair(dsf, ds, s2);
#pragma unroll
        for (int c = 0; c < NCT; ++c) {
          const int n = s2 * NCT + c;
          mfma16(acc_dv[c], ot2[n % AHEAD], pf);   // dV^T[c][j]
          mfma16(acc_dk[c], qt2[n % AHEAD], dsf);  // dK^T[c][j]
          if (n + AHEAD < 2 * NCT) {
            trfrag(ot2[n % AHEAD], ost, (n + AHEAD) / NCT, (n + AHEAD) % NCT);
            trfrag(qt2[n % AHEAD], qst, (n + AHEAD) / NCT, (n + AHEAD) % NCT);
          }
        }
      }
    }
    if (more) store_rows(cur ^ 1);
  }

  auto sums = [&](int c, float (&vk)[4], float (&vv)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      vk[i] = kj < n_keys ? acc_dk[c][i] * a.scale : 0.f;  // (padding: zeros)
      vv[i] = kj < n_keys ? acc_dv[c][i] : 0.f;
    }
  };
  if (ranges) {
    if (kj >= n_keys) return;
    const int64_t r = (static_cast<int64_t>(split) * BH + bh) * a.Tk + kj;
#pragma unroll
    for (int c = 0; c < NCT; ++c) {
      float vk[4], vv[4];
      sums(c, vk, vv);
      store_row4<float>(a.part_k + r * DH + c * 16 + 4 * lg, vk);
      store_row4<float>(a.part_v + r * DH + c * 16 + 4 * lg, vv);
    }
    return;
  }
  Rows<DH, 16> out{lds + w * 2 * 16 * RB}, out_v{lds + (w * 2 + 1) * 16 * RB};
  stages_done();
#pragma unroll
  for (int c = 0; c < NCT; ++c) {
    float vk[4], vv[4];
    sums(c, vk, vv);
    out.put(lr, c, lg, vk);
    out_v.put(lr, c, lg, vv);
  }
  const int k_end = a.k_start ? n_keys : a.Tk;
  bf16_t *dk = static_cast<bf16_t*>(a.dk) + ks.row0 * a.lddk + hk * DH, *dv = static_cast<bf16_t*>(a.dv) + ks.row0 * a.lddv + hk * DH;
  out.store(lane, [&](int row, bool& on) { return on = kw + row < k_end, dk + (kw + row) * a.lddk; });
  out_v.store(lane, [&](int row, bool& on) { return on = kw + row < k_end, dv + (kw + row) * a.lddv; });
}

// Large problems: a launch each.  dQ in workgroups of four waves of 16 or 32 queries,
// dK and dV of eight waves of 16 keys, two tiles a barrier.
template <int DH, int GR>
__global__ void __launch_bounds__(256, 2) cross_dq_kernel(const CrossArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * FwdDL<DH>::STAGE];
  const int item = item_of(a.n_x * a.B * a.Hk * a.splits, blockIdx.x);
  if (item >= 0) dq_body<DH, GR, 4>(lds, a, item);
}
template <int DH>
__global__ void __launch_bounds__(512, DH == 64 ? 4 : 2) cross_dkdv_kernel(const CrossArgs a) {
  constexpr int SUB = 2;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * SUB * dkdv_stage<DH>()];
  const int item = item_of(a.k_x * a.B * a.Hk * a.k_splits, blockIdx.x);
  if (item >= 0) dkdv_body<DH, 8, SUB, false>(lds, nullptr, a, item);
}

// Small ones: both in one launch, workgroups of 64 rows, D computed on both
// sides, so that neither waits for the other and twice as many CUs have work
// (packed 333, 255 and 270 queries of 16 heads on 200, 39 and 108 keys of 4 heads of
// 128: 34.8 us in two launches, 27 in one).
template <int DH>
__global__ void __launch_bounds__(256, DH == 64 ? 3 : 2) cross_bwd_small_kernel(const CrossArgs a) {
  constexpr int STAGES = 2 * dkdv_stage<DH>();
  static_assert(dkdv_stage<DH>() >= FwdDL<DH>::STAGE, "stages");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[STAGES + SMALL_ROWS * 4];
  // the first part of the grid dK and dV, the rest dQ: every XCD has both
  const int n_k = a.dk ? a.k_x * a.B * a.Hk * a.k_splits : 0, n_q = a.dq ? a.n_x * a.B * a.Hk * a.splits : 0;
  const int k_end = (n_k + 7) & ~7, id = blockIdx.x;
  const int item = id < k_end ? item_of(n_k, id) : item_of(n_q, id - k_end);
  if (item < 0) return;
  if (id < k_end) dkdv_body<DH, 4, 1, true>(lds, reinterpret_cast<float*>(lds + STAGES), a, item);
  else dq_body<DH, 1, 4>(lds, a, item);
}

}  // namespace cross

namespace {

using namespace cross;

// The shape of each launch: blocks of rows, ranges, and the workspace.
struct Plan {
  int blk;  // rows of a workgroup: 64, 128 or 256
  int n_x, splits;
};

constexpr int64_t CUS = 256;
// What a launch takes, in us, for the choice of its workgroups' rows and ranges: a
// workgroup that has its CU to itself takes start + tile for each tile of the other
// side, w of them on a CU share w times as much (where several fit; where one does,
// they follow each other), and a last round that leaves most CUs idle takes `last`
// of a full one.  Measured with all CUs busy, and rounded.  (us, heads of 128, forward
// in 256-row and in 128-row workgroups: 2048 x 1024, 32 heads 45.7 and 46.0, 40: 68.9
// and 58.1, 56: 73.7 and 73.5; 20,000 x 300, 16 heads 95 and 84; 2 x 2048 x 4096, 32
// heads 266 and 276.  Heads of 64, 128 and 64 rows: 8 x 300 x 1500, 12 heads 37 and 27;
// 8 x 1024 x 1024 38 and 42.  Gradients with dQ in 128 and 64 rows: 8 x 300 x 1500, 12
// heads of 64, 81 and 69; 8 x 128 x 1500, 16 heads of 128, 113 and 107, 2 x 2048 x 4096, 32
// heads 923 and 1017; 2 x 2048 x 1500, 32 heads 360, in 256 rows 367.  fp32, one range
// of 16 and of 32 tiles, 256 workgroups: heads of 64 and of 128, forward 60 and 103, 102
// and 195, dQ 73 and 139, 141 and 270; 512 workgroups 32 tiles 183, 344, 239, 458.  dK
// and dV, with the pass for D, 148 and 293, 366 and 679, 512 workgroups 489 and 1087: a
// tile takes a third more than its row says.  Two ranges, 256 workgroups: 139 and 266,
// 320 and 567, taken by these figures but for the first.)
struct Cost {
  int blk;  // rows; 0: no such kernel
  double tile, start, share, last;
};
using Costs = Cost[3];
constexpr Costs FWD[2] = {{{64, 0.45, 1.2, 0.78, 0.55}, {128, 0.76, 1.8, 0.77, 0.55}, {}},
                          {{64, 0.92, 2.0, 0.76, 0.55}, {128, 1.28, 2.75, 0.91, 0.55}, {256, 2.2, 7.5, 1.0, 0.55}}};
constexpr Costs DQ[2] = {{{64, 0.68, 1.3, 0.80, 0.55}, {128, 1.15, 2.0, 0.77, 0.55}, {}},
                         {{64, 1.15, 2.5, 0.85, 0.55}, {128, 1.6, 3.0, 0.94, 0.55}, {}}};
constexpr Costs DKDV[2] = {{{128, 1.5, 3.0, 0.77, 0.55}, {}, {}}, {{128, 1.9, 6.0, 1.0, 0.8}, {}, {}}};
constexpr Costs FWD_F32[2] = {{{64, 2.7, 2.0, 0.8, 0.55}, {}, {}}, {{64, 5.3, 2.0, 0.8, 0.55}, {}, {}}};
constexpr Costs DQ_F32[2] = {{{64, 4.0, 3.0, 0.8, 0.55}, {}, {}}, {{64, 8.0, 3.0, 0.8, 0.55}, {}, {}}};
constexpr Costs DKDV_F32[2] = {{{64, 5.0, 3.0, 0.8, 0.55}, {}, {}}, {{64, 10.0, 3.0, 0.8, 0.55}, {}, {}}};
// Ranges cost a launch that joins their sums, and the way of those to memory and
// back, by the 1000 numbers that each CU has.  (4 x 300 x 500, 12 heads of 64, 240
// workgroups: 10.3 us, in two ranges 20.0; 2 x 512 x 16000, 8 heads of 128, 32 of 256
// rows: 415, in 8 ranges 84, in 12 105; 20,000 x 300, 16 heads, gradients: 713 with one
// range of queries, 281 with five, which fill a round of CUs, 340 with six.)
constexpr double JOIN = 8.0, JOIN_KILO = 0.15;
// More ranges have to be faster by this (8 x 128 x 1500, 16 heads of 64, gradients: dQ
// in two ranges 59 us, in four, the same by these figures, 63).
constexpr double GAIN = 0.95;

// Blocks of `rows` rows of `heads` heads over `tiles` tiles, `width` numbers in a
// row's sums: the kernel and the ranges (as many as fit one to four workgroups a
// CU) that take least.
Plan plan_of(const Costs& kernels, int64_t rows, int64_t heads, int64_t tiles, int width) {
  Plan best{};
  double least = 0;
  for (const Cost& c : kernels) {
    if (!c.blk) continue;
    const int64_t n_x = (rows + c.blk - 1) / c.blk, n = n_x * heads;
    int64_t splits = 0;
    double mine = 0;
    for (int64_t k = 0; k <= 4; ++k) {
      if (k && k * CUS < 2 * n) continue;
      const int64_t s = k == 0 || n == 0 ? 1 : std::min(k * CUS / n, tiles / 2);
      if (k && s <= 1) continue;
      const int64_t rem = n * s % CUS;
      const double w = std::max(1.0, static_cast<double>(n * s / CUS) + (rem ? std::max(c.last, 1.0 * rem / CUS) : 0.0));
      double t = std::max(1.0, c.share * w) * (c.tile * ((tiles + s - 1) / s) + c.start);
      if (s > 1) t += JOIN + JOIN_KILO * 1e-3 * w * c.blk * width;
      if (splits == 0 || t < GAIN * mine) splits = s, mine = t;
    }
    if (best.blk == 0 || mine < least) best = Plan{c.blk, static_cast<int>(n_x), static_cast<int>(splits)}, least = mine;
  }
  return best;
}
// Tiles of 64 x 64 for each of two workgroups a CU, of both sides, up to which
// the backward is one launch.  In two launches and in one, us: heads of 128, 8
// tiles (2 x 512 x 512, 16 heads) 47 and 34, 12 tiles 44 and 48 (3 x 512 x 512), 55
// and 52 (1000 x 333, 32 heads), 16 tiles 49 and 59, 32 tiles 75 and 100; heads of
// 64, 16 tiles 28 and 34, 22 to 24 tiles 46 and 43, 47 and 45.
constexpr int64_t SMALL_TILES_64 = 12, SMALL_TILES_128 = 8;
// Tiles that ranges have to save a workgroup of a small backward, to be worth their
// join's launch (1 to 6 measured the same).
constexpr int64_t RANGE_GAIN = 2;

// One block of rows for each sequence and head is a call that reads its keys for
// little work (single tokens): it takes more ranges, so that many loads are in
// flight and long sequences do not wait for one workgroup.  (Workgroups wanted, and
// tiles of keys a range has at least, us of 8 x 1 x 2048 of 40 heads of 128, ragged,
// and of 16 x 1 x 4000 of 32 heads on 4: one range 72, -; 1024, 8: 52.3, 33.4; 1024,
// 4: 52.5, 39.1; 2048, 4: 53.8, 39.3; 2048, 2: 53.8, 48.7; 4096, 2: 61.7, 49.0.  Both
// shapes have the card full.  One sequence of few heads has not, and its workgroups
// still walk eight tiles: one token of 32 heads of 128 on 2048 keys of 8 heads, 32
// workgroups, 13.5 us, fp32 26; fewer tiles a range are not measured there.)
constexpr int64_t TOKEN_WGS = 1024, TOKEN_TILES = 8;

Plan fwd_plan(int dtype, int B, int Tq, int Tk, int Hk, int G, int dh) {
  const int64_t rows = static_cast<int64_t>(Tq) * G, heads = static_cast<int64_t>(B) * Hk;
  const int64_t tiles = (Tk + attn::BT - 1) / attn::BT;
  if (rows <= 64) {
    const int64_t s = heads > 0 ? std::min<int64_t>(TOKEN_WGS / heads, tiles / TOKEN_TILES) : 1;
    return Plan{64, static_cast<int>((rows + 63) / 64), static_cast<int>(std::max<int64_t>(1, s))};
  }
  return plan_of(dtype == DT_BF16 ? FWD[dh == 128] : FWD_F32[dh == 128], rows, heads, tiles, dh);
}
// The backward's two sides: q (blocks of queries, ranges of keys) and k.
struct BwdPlan {
  bool small;
  Plan q, k;
};
// Ranges of a side that bring a workgroup's tiles from `all` to the `fair` share, but
// not below `least`; none where that saves RANGE_GAIN tiles or fewer.
int ranges_of(int64_t all, int64_t fair, int64_t least) {
  const int64_t per = std::max(fair, least);
  return static_cast<int>(all > per + RANGE_GAIN ? (all + per - 1) / per : 1);
}
BwdPlan bwd_plan(int dtype, int B, int Tq, int Tk, int Hk, int G, int dh) {
  const int64_t heads = static_cast<int64_t>(B) * Hk, rows = static_cast<int64_t>(Tq) * G;
  const int64_t tq = (rows + attn::BT - 1) / attn::BT, tk = (Tk + attn::BT - 1) / attn::BT;
  BwdPlan p{};
  const int64_t fair = (2 * tq * tk * heads + 2 * CUS - 1) / (2 * CUS);
  p.small = fair <= (dh == 64 ? SMALL_TILES_64 : SMALL_TILES_128);
  if (p.small) {
    // both sides share two workgroups a CU
    p.q = Plan{64, static_cast<int>(tq), ranges_of(tk, fair, 2)};
    // (and D of a range of queries has to fit the LDS)
    p.k = Plan{64, static_cast<int>(tk),
               std::max(ranges_of(tq, fair, 2), static_cast<int>((tq + SMALL_ROWS / attn::BT - 1) / (SMALL_ROWS / attn::BT)))};
  } else {
    p.q = plan_of(dtype == DT_BF16 ? DQ[dh == 128] : DQ_F32[dh == 128], rows, heads, tk, dh);
    p.k = plan_of(dtype == DT_BF16 ? DKDV[dh == 128] : DKDV_F32[dh == 128], Tk, heads, tq, 2 * dh);
  }
  return p;
}

// Grids are multiples of eight (see item_of).
unsigned grid_of(const CrossArgs& a, int64_t x, int64_t splits) {
  return static_cast<unsigned>((x * splits * a.B * a.Hk + 7) / 8 * 8);
}

// Sums of the ranges to dq (packed rows, times the scale) and to dk and dv (which
// hold it), a side that has none left out: W waves a row, each every W-th range in
// order, then the waves in order.
template <typename T, int DH, int W>
__global__ void __launch_bounds__(W == 1 ? 256 : 64 * W) cross_sum_kernel(const CrossArgs a, int64_t n_q, int64_t n_k) {
  constexpr int E = DH / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = W == 1 ? 0 : wave;
  int64_t r = W == 1 ? static_cast<int64_t>(blockIdx.x) * 4 + wave : blockIdx.x;
  const bool q_side = r < n_q;
  if (!q_side) r -= n_q;
  const int64_t n = q_side ? n_q : n_k, per = q_side ? static_cast<int64_t>(a.Tq) * a.G : a.Tk;
  if (r >= n) return;
  const int bh = static_cast<int>(r / per), i = static_cast<int>(r % per), b = bh % a.B, hk = bh / a.B;
  const Seq s = q_side ? seq(a.q_start, a.q_len, a.Tq, a.q_rows, b) : seq(a.k_start, a.k_len, a.Tk, a.k_rows, b);
  const bool on = i < (q_side ? s.n * a.G : s.n);
  if (!on && (q_side ? a.q_start : a.k_start)) return;
  const int splits = !on ? 0 : q_side ? a.splits : a.k_splits;
  float v[2][E] = {};
  const int64_t at_r = (first * n + r) * DH + E * lane, step = W * n * DH;
  if (q_side) {
    const float* p = a.part + at_r;
#pragma unroll 8
    for (int j = first; j < splits; j += W, p += step)
#pragma unroll
      for (int e = 0; e < E; ++e) v[0][e] += p[e];
  } else {
    const float *pk = a.part_k + at_r, *pv = a.part_v + at_r;
#pragma unroll 8
    for (int j = first; j < splits; j += W, pk += step, pv += step)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[0][e] += pk[e];
        v[1][e] += pv[e];
      }
  }
  if constexpr (W > 1) {
    __shared__ float sums[W][64][2 * E];
#pragma unroll
    for (int e = 0; e < 2 * E; ++e) sums[wave][lane][e] = v[e / E][e % E];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < W; ++w)
#pragma unroll
      for (int e = 0; e < 2 * E; ++e) v[e / E][e % E] += sums[w][lane][e];
  }
  if (q_side) {
    const int64_t lo = at<DH>(a, s, hk, i, a.lddq) + E * lane;
#pragma unroll
    for (int e = 0; e < E; ++e) static_cast<T*>(a.dq)[lo + e] = from_f<T>(v[0][e] * a.scale);
  } else {
    const int64_t row = s.row0 + i, col = hk * DH + E * lane;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      static_cast<T*>(a.dk)[row * a.lddk + col + e] = from_f<T>(v[0][e]);
      static_cast<T*>(a.dv)[row * a.lddv + col + e] = from_f<T>(v[1][e]);
    }
  }
}

template <int DH, int GR, int NW>
void fwd_launch(const CrossArgs& a, hipStream_t s) {
  const dim3 grid(grid_of(a, a.n_x, a.splits)), block(64 * NW);
  if (a.splits > 1) hipLaunchKernelGGL((cross_fwd_kernel<DH, GR, NW, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((cross_fwd_kernel<DH, GR, NW, false>), grid, block, 0, s, a);
}
hipError_t fwd_bf16(const CrossArgs& a, int blk, int dh, hipStream_t s) {
  if (dh == 64) {
    if (blk == 64) fwd_launch<64, 1, 4>(a, s);
    else fwd_launch<64, 2, 4>(a, s);
  } else {
    if (blk == 64) fwd_launch<128, 1, 4>(a, s);
    else if (blk == 128) fwd_launch<128, 2, 4>(a, s);
    else fwd_launch<128, 2, 8>(a, s);
  }
  return hipGetLastError();
}

unsigned rows_grid(int64_t rows) { return static_cast<unsigned>((rows + 3) / 4); }

// Ranges from which a row's sums are joined by JOIN_WAVES waves (one token of 32 heads
// on 100,000 keys of 4, 195 ranges: 100 us by one wave, serially; 11).
constexpr int JOIN_WIDE = 16, JOIN_WAVES = 8;
constexpr int64_t JOIN_ROWS = 1 << 14;  // (more rows fill the card with a wave each)
template <typename T, int DH>
void join_launch(const CrossArgs& a, int64_t rows, hipStream_t s) {
  if (a.splits >= JOIN_WIDE && rows <= JOIN_ROWS)
    hipLaunchKernelGGL((cross_join_kernel<T, DH, JOIN_WAVES>), dim3(static_cast<unsigned>(rows)), dim3(64 * JOIN_WAVES), 0, s, a);
  else hipLaunchKernelGGL((cross_join_kernel<T, DH, 1>), dim3(rows_grid(rows)), dim3(256), 0, s, a);
}
template <typename T>
hipError_t join(const CrossArgs& a, int dh, hipStream_t s) {
  const int64_t rows = static_cast<int64_t>(a.Tq) * a.G * a.B * a.Hk;
  if (dh == 64) join_launch<T, 64>(a, rows, s);
  else join_launch<T, 128>(a, rows, s);
  return hipGetLastError();
}

template <int DH>
hipError_t bwd_bf16(const CrossArgs& a, const BwdPlan& p, hipStream_t s) {
  const unsigned nq = a.dq || a.delta ? grid_of(a, a.n_x, a.splits) : 0, nk = a.dk ? grid_of(a, a.k_x, a.k_splits) : 0;
  if (p.small) {
    if (nq + nk) hipLaunchKernelGGL(cross_bwd_small_kernel<DH>, dim3(nq + nk), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  // dQ first: it computes D
  if (nq) {
    if (p.q.blk == 128) hipLaunchKernelGGL((cross_dq_kernel<DH, 2>), dim3(nq), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cross_dq_kernel<DH, 1>), dim3(nq), dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (nk) hipLaunchKernelGGL(cross_dkdv_kernel<DH>, dim3(nk), dim3(512), 0, s, a);
  return hipGetLastError();
}

template <typename T, int DH>
void sum_launch(const CrossArgs& a, int64_t n_q, int64_t n_k, hipStream_t s) {
  const int64_t rows = n_q + n_k;
  // (a side that has no ranges has no rows here)
  if (std::max(n_q ? a.splits : 0, n_k ? a.k_splits : 0) >= JOIN_WIDE && rows <= JOIN_ROWS)
    hipLaunchKernelGGL((cross_sum_kernel<T, DH, JOIN_WAVES>), dim3(static_cast<unsigned>(rows)), dim3(64 * JOIN_WAVES), 0, s, a, n_q, n_k);
  else hipLaunchKernelGGL((cross_sum_kernel<T, DH, 1>), dim3(rows_grid(rows)), dim3(256), 0, s, a, n_q, n_k);
}
template <typename T>
hipError_t sum(const CrossArgs& a, int dh, hipStream_t s) {
  const int64_t heads = static_cast<int64_t>(a.B) * a.Hk;
  const int64_t n_q = a.dq && a.splits > 1 ? a.Tq * heads * a.G : 0, n_k = a.dk && a.k_splits > 1 ? a.Tk * heads : 0;
  if (n_q + n_k == 0) return hipSuccess;
  if (dh == 64) sum_launch<T, 64>(a, n_q, n_k, s);
  else sum_launch<T, 128>(a, n_q, n_k, s);
  return hipGetLastError();
}

// Floats of a ws, in whole 16-byte pieces.
uint64_t up4(uint64_t n) { return (n + 3) / 4 * 4; }

}  // namespace

bool cross_attn_ok(int B, int Tq, int Tk, int Hq, int Hk, int dh) {
  if (B < 0 || Tq < 0 || Tk < 0 || Hq < 1 || Hk < 1 || Hq % Hk || (dh != 64 && dh != 128)) return false;
  const int64_t G = Hq / Hk, heads = static_cast<int64_t>(B) * Hk;
  // (row_of's products)
  if (Tq > 0 && (G >= 1 << 16 || Tq * G * G >= 1ll << 32)) return false;
  if (Tq * G >= 1ll << 30 || Tk >= 1 << 30 || heads >= 1 << 30) return false;
  // rows of the launches that join ranges, four a workgroup
  if (heads * (Tq * G + Tk) >= MAX_WORKGROUPS * 4 - 4) return false;
  // Workgroups of either call, below half of what a dispatch counts (512 threads
  // each): of 64 rows, or where ranges multiply them, a few thousand.
  const int64_t n = ((Tq * G + 63) / 64 + (Tk + 63) / 64) * heads;
  return n + (1 << 14) < MAX_WORKGROUPS / 2;
}

uint64_t cross_attn_fwd_ws(int dtype, int B, int Tq, int Tk, int Hq, int Hk, int dh) {
  const Plan p = fwd_plan(dtype, B, Tq, Tk, Hk, Hq / Hk, dh);
  if (p.splits == 1) return 0;
  const uint64_t rows = static_cast<uint64_t>(p.splits) * B * Hq * Tq;
  return 4 * (rows * dh + up4(2 * rows));
}

// Floats of the backward's workspace: D (large problems), then the ranges' sums.
struct BwdSpace {
  uint64_t delta, q, k;
};
static BwdSpace bwd_space(const BwdPlan& p, int64_t rows_q, int64_t rows_k, int dh) {
  BwdSpace s{};
  s.delta = p.small ? 0 : up4(rows_q);
  s.q = p.q.splits > 1 ? static_cast<uint64_t>(p.q.splits) * rows_q * dh : 0;
  s.k = p.k.splits > 1 ? static_cast<uint64_t>(p.k.splits) * rows_k * dh : 0;
  return s;
}

uint64_t cross_attn_bwd_ws(int dtype, int B, int Tq, int Tk, int Hq, int Hk, int dh) {
  const BwdSpace w = bwd_space(bwd_plan(dtype, B, Tq, Tk, Hk, Hq / Hk, dh), static_cast<int64_t>(Hq) * B * Tq,
                               static_cast<int64_t>(B) * Hk * Tk, dh);
  return 4 * (w.delta + w.q + 2 * w.k);
}

hipError_t cross_attn_fwd(int dtype, CrossArgs& a, int dh, void* ws, hipStream_t s) {
  const Plan p = fwd_plan(dtype, a.B, a.Tq, a.Tk, a.Hk, a.G, dh);
  a.n_x = p.n_x, a.splits = p.splits;
  if (a.splits > 1) {
    a.part = static_cast<float*>(ws);
    a.ml = a.part + static_cast<uint64_t>(p.splits) * a.B * a.Hq * a.Tq * dh;
  }
  hipError_t e;
  if (dtype == DT_BF16) {
    e = fwd_bf16(a, p.blk, dh, s);
  } else {
    e = cross_fwd_f32(a, dh, s);
  }
  if (e != hipSuccess || a.splits == 1) return e;
  return dtype == DT_BF16 ? join<bf16_t>(a, dh, s) : join<float>(a, dh, s);
}

hipError_t cross_attn_bwd(int dtype, CrossArgs& a, int dh, void* ws, hipStream_t s) {
  const BwdPlan p = bwd_plan(dtype, a.B, a.Tq, a.Tk, a.Hk, a.G, dh);
  const BwdSpace w = bwd_space(p, static_cast<int64_t>(a.Hq) * a.B * a.Tq, static_cast<int64_t>(a.B) * a.Hk * a.Tk, dh);
  float* f = static_cast<float*>(ws);
  a.delta = p.small ? nullptr : f;
  a.part = f + w.delta, a.part_k = a.part + w.q, a.part_v = a.part_k + w.k;
  a.n_x = p.q.n_x, a.splits = a.dq ? p.q.splits : 1;
  a.k_x = p.k.n_x, a.k_splits = p.k.splits;
  if (a.Tq == 0) a.dq = nullptr, a.delta = nullptr;
  if (a.Tk == 0) a.dk = a.dv = nullptr;
  hipError_t e;
  if (dtype != DT_BF16) e = cross_bwd_f32(a, dh, p.small, s);
  else e = dh == 64 ? bwd_bf16<64>(a, p, s) : bwd_bf16<128>(a, p, s);
  if (e != hipSuccess) return e;
  return dtype == DT_BF16 ? sum<bf16_t>(a, dh, s) : sum<float>(a, dh, s);
}

}  // namespace atom
