// Cross attention in fp32 (validation mode): the tiles of cross_attention.hip on
// fp32 matrix instructions.  Workgroups of four waves, 16 rows each; tiles of 64
// rows in their natural layout, through registers into padded LDS, two stages.
// A transposed operand is read by elements: a fragment's eight matrix
// instructions take 256 cycles, its eight LDS reads 16.  2 x 512 x 512, 16 heads of
// 128: 50 us forward, 150 backward (86 and, with the scores and dP that are computed
// twice, 100 TFLOP/s; a library product 142).  dK and dV at heads of 128 need more than
// 256 registers, two tiles on their way to LDS beside K, V and both sums: 84 are
// spilled, 78 in the small backward.
#include "cross_attention.h"

namespace atom {
namespace cross {

using namespace attn;

template <int DH>
struct Tile {
  static constexpr int RP = DH + 4;            // pitch of a row
  static constexpr int N = BT * DH / 4 / 256;  // 16-byte chunks of a thread
  f32x4_t r[N];
  // rows r0 .. of the list that `addr` maps to addresses; behind the last (n
  // of them, at least one) the last again
  template <typename F>
  ATOM_DEV void load(F addr, int r0, int n, int tid) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = i * 256 + tid;
      r[i] = *reinterpret_cast<const f32x4_t*>(addr(min(r0 + id / (DH / 4), n - 1)) + id % (DH / 4) * 4);
    }
  }
  ATOM_DEV void store(float* s, int tid) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = i * 256 + tid;
      *reinterpret_cast<f32x4_t*>(s + id / (DH / 4) * RP + id % (DH / 4) * 4) = r[i];
    }
  }
  // rows of 32 columns from 32 s on, and column c of the rows that frag_from_pair
  // gives eight elements
  static ATOM_DEV void row(Frag<float>& f, const float* s, int r, int col) { frag_load(f, s + r * RP + col); }
  static ATOM_DEV void col(Frag<float>& f, const float* s, int c, int s2, int lg) {
    const float* p = s + (32 * s2 + 4 * lg) * RP + c;
    f.lo = make_float4(p[0], p[RP], p[2 * RP], p[3 * RP]);
    p += 16 * RP;
    f.hi = make_float4(p[0], p[RP], p[2 * RP], p[3 * RP]);
  }
};

// Scores are sums of DH terms; each of two accumulators takes half of them, so
// that fewer roundings meet the large partial sums (an instruction rounds after
// each of its four products), and the instructions' chains are half as long.
struct Halves {
  f32x4_t x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  ATOM_DEV void add(int s, const Frag<float>& a, const Frag<float>& b) { mfma16(x[s & 1], a, b); }
  ATOM_DEV f32x4_t sum() const { return x[0] + x[1]; }
};

struct Item {
  int x, split, bh, b, hk;
};
ATOM_DEV Item item(const CrossArgs& a, int i, int n_x, int splits) {
  const int bh = i / (n_x * splits);
  return Item{i % n_x, i / n_x % splits, bh, bh % a.B, bh / a.B};
}

ATOM_DEV void range_of(int n_rows, int splits, int s, int* t0, int* t1) {
  const int n = (n_rows + BT - 1) / BT, per = (n + splits - 1) / splits;
  *t0 = min(s * per, n);
  *t1 = min(s * per + per, n);
}

// FEW: at most 16 rows (single tokens), which all four waves share, each taking
// 16 of a tile's 64 keys; their sums meet at the end (8 x 2000 keys, 16 heads of
// 128: 153 us with one wave at work, see the launcher).
template <int DH, bool FEW>
__global__ void __launch_bounds__(256, 2) cross_fwd_f32_kernel(const CrossArgs a) {
  using L = Tile<DH>;
  static_assert(!FEW || 3 * 64 * (DH / 4 + 2) <= BT * L::RP, "the waves' sums in a tile's place");
  constexpr int NS = DH / 32, NCT = DH / 16;
  constexpr int JT = FEW ? 1 : 4;  // 16-key parts of a tile that a wave takes
  __shared__ __attribute__((aligned(16))) float Ks[BT * L::RP], Vs[BT * L::RP];
  const int id = item_of(a.n_x * a.B * a.Hk * a.splits, blockIdx.x);
  if (id < 0) return;
  const Item it = item(a, id, a.n_x, a.splits);
  const Seq qs = seq(a.q_start, a.q_len, a.Tq, a.q_rows, it.b), ks = seq(a.k_start, a.k_len, a.Tk, a.k_rows, it.b);
  const int P = qs.n * a.G, q0 = it.x * 64, hk = it.hk;
  if (q0 >= P && (a.splits > 1 || a.q_start)) return;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lr = lane & 15, lg = lane >> 4;
  const int pi = q0 + (FEW ? 0 : w * 16) + lr, j_w = FEW ? w * 16 : 0;
  const float* kb = static_cast<const float*>(a.k) + ks.row0 * a.ldk + hk * DH;
  const float* vb = static_cast<const float*>(a.v) + ks.row0 * a.ldv + hk * DH;
  auto k_at = [&](int j) { return kb + j * a.ldk; };
  auto v_at = [&](int j) { return vb + j * a.ldv; };

  Frag<float> qf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    if (pi < P) frag_load(qf[s], static_cast<const float*>(a.q) + at<DH>(a, qs, hk, pi, a.ldq) + 32 * s + 8 * lg);
    else frag_zero(qf[s]);
  }
  f32x4_t acc[NCT];
#pragma unroll
  for (int c = 0; c < NCT; ++c) acc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = NO_MAX, l = 0.f;

  int t0 = 0, t1 = 0;
  if (q0 < P) range_of(ks.n, a.splits, it.split, &t0, &t1);
  L lk, lv;
  if (t0 < t1) {
    lk.load(k_at, t0 * BT, ks.n, tid);
    lv.load(v_at, t0 * BT, ks.n, tid);
  }
  for (int kt = t0; kt < t1; ++kt) {
    __syncthreads();
    lk.store(Ks, tid);
    lv.store(Vs, tid);
    __syncthreads();
    if (kt + 1 < t1) {
      lk.load(k_at, (kt + 1) * BT, ks.n, tid);
      lv.load(v_at, (kt + 1) * BT, ks.n, tid);
    }
    float p[JT][4], mx = -INFINITY;
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) {
      Halves zh;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        Frag<float> kf;
        L::row(kf, Ks, j_w + jt * 16 + lr, 32 * s + 8 * lg);
        zh.add(s, kf, qf[s]);
      }
      const f32x4_t z = zh.sum();
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[jt][r] = kt * BT + j_w + jt * 16 + 4 * lg + r < ks.n ? z[r] : -INFINITY;
        mx = fmaxf(mx, p[jt][r]);
      }
    }
    const float m_new = fmaxf(m, rows4_max(mx) * a.scale), alpha = exp_near(m - m_new);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int c = 0; c < NCT; ++c) acc[c] *= alpha;
#pragma unroll
    for (int jt = 0; jt < JT; ++jt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[jt][r] = exp_near(__builtin_fmaf(p[jt][r], a.scale, -m));
        l += p[jt][r];
      }
    if constexpr (FEW) {
      const float* vp = Vs + (j_w + 4 * lg) * L::RP + lr;
#pragma unroll
      for (int c = 0; c < NCT; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vp[r * L::RP + c * 16], p[0][r], acc[c], 0, 0, 0);
    } else {
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        Frag<float> pf;
        frag_from_pair(pf, p, s2);
#pragma unroll
        for (int c = 0; c < NCT; ++c) {
          Frag<float> vf;
          L::col(vf, Vs, c * 16 + lr, s2, lg);
          mfma16(acc[c], vf, pf);
        }
      }
    }
  }

  float l_tot = rows4_sum(l);
  if constexpr (FEW) {
    // the waves' sums, brought to the largest maximum, in wave order
    float* sums = Ks;
    __syncthreads();
    if (w) {
      float* mine = sums + ((w - 1) * 64 + lane) * (4 * NCT + 2);
#pragma unroll
      for (int c = 0; c < NCT; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) mine[4 * c + r] = acc[c][r];
      mine[4 * NCT] = m;
      mine[4 * NCT + 1] = l_tot;
    }
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int v = 0; v < 3; ++v) {
      const float* o = sums + (v * 64 + lane) * (4 * NCT + 2);
      const float m1 = fmaxf(m, o[4 * NCT]), f0 = exp_near(m - m1), f1 = exp_near(o[4 * NCT] - m1);
      m = m1;
      l_tot = l_tot * f0 + o[4 * NCT + 1] * f1;
#pragma unroll
      for (int c = 0; c < NCT; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[c][r] = acc[c][r] * f0 + o[4 * c + r] * f1;
    }
  }
  const int64_t n_p = static_cast<int64_t>(a.Tq) * a.G;
  if (a.splits > 1) {
    if (pi >= P) return;
    const int64_t r = (static_cast<int64_t>(it.split) * a.B * a.Hk + it.bh) * n_p + pi;
#pragma unroll
    for (int c = 0; c < NCT; ++c) {
      float v[4] = {acc[c][0], acc[c][1], acc[c][2], acc[c][3]};
      store_row4<float>(a.part + r * DH + c * 16 + 4 * lg, v);
    }
    if (lg == 0) a.ml[2 * r] = m, a.ml[2 * r + 1] = l_tot;
    return;
  }
  if (pi >= (a.q_start ? P : n_p)) return;
  const bool none = l_tot == 0.f || pi >= P;  // no keys, or padding: zeros
  const float inv = 1.f / l_tot;
  float* orow = static_cast<float*>(a.o) + at<DH>(a, qs, hk, pi, a.ldo);
#pragma unroll
  for (int c = 0; c < NCT; ++c) {
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = none ? 0.f : acc[c][r] * inv;
    store_row4<float>(orow + c * 16 + 4 * lg, v);
  }
  if (lg == 0 && a.lse) {
    const Row rw = row_of(a, pi);
    a.lse[(qs.row0 + rw.t) * a.Hq + hk * a.G + rw.g] = none ? -INFINITY : m + logf(l_tot);
  }
}

// dQ, and D of every row (a.dq null: D alone).
template <int DH>
ATOM_DEV void dq_f32(float* Ks, float* Vs, const CrossArgs& a, int id) {
  using L = Tile<DH>;
  constexpr int NS = DH / 32, NCT = DH / 16;
  const Item it = item(a, id, a.n_x, a.splits);
  const Seq qs = seq(a.q_start, a.q_len, a.Tq, a.q_rows, it.b), ks = seq(a.k_start, a.k_len, a.Tk, a.k_rows, it.b);
  const int P = qs.n * a.G, q0 = it.x * 64, hk = it.hk;
  if (q0 >= P && (a.splits > 1 || a.q_start)) return;
  const int64_t n_p = static_cast<int64_t>(a.Tq) * a.G;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lr = lane & 15, lg = lane >> 4;
  const int pi = q0 + w * 16 + lr;
  const float* kb = static_cast<const float*>(a.k) + ks.row0 * a.ldk + hk * DH;
  const float* vb = static_cast<const float*>(a.v) + ks.row0 * a.ldv + hk * DH;
  auto k_at = [&](int j) { return kb + j * a.ldk; };
  auto v_at = [&](int j) { return vb + j * a.ldv; };

  Frag<float> qf[NS], of[NS];
  float lse_i = INFINITY, del = 0.f;
  if (pi < P) {
    const Row rw = row_of(a, pi);
    lse_i = lse_of(a.lse[(qs.row0 + rw.t) * a.Hq + hk * a.G + rw.g]);
  }
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    frag_zero(qf[s]);
    frag_zero(of[s]);
    if (pi < P) {
      Frag<float> f;
      frag_load(qf[s], static_cast<const float*>(a.q) + at<DH>(a, qs, hk, pi, a.ldq) + 32 * s + 8 * lg);
      frag_load(of[s], static_cast<const float*>(a.dout) + at<DH>(a, qs, hk, pi, a.lddo) + 32 * s + 8 * lg);
      frag_load(f, static_cast<const float*>(a.o) + at<DH>(a, qs, hk, pi, a.ldo) + 32 * s + 8 * lg);
      del += f.lo.x * of[s].lo.x + f.lo.y * of[s].lo.y + f.lo.z * of[s].lo.z + f.lo.w * of[s].lo.w;
      del += f.hi.x * of[s].hi.x + f.hi.y * of[s].hi.y + f.hi.z * of[s].hi.z + f.hi.w * of[s].hi.w;
    }
  }
  del = rows4_sum(del);
  if (a.delta && lg == 0 && pi < P && it.split == 0) a.delta[it.bh * n_p + pi] = del;
  if (!a.dq) return;
  f32x4_t acc[NCT];
#pragma unroll
  for (int c = 0; c < NCT; ++c) acc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  int t0 = 0, t1 = 0;
  if (q0 < P) range_of(ks.n, a.splits, it.split, &t0, &t1);
  L lk, lv;
  if (t0 < t1) {
    lk.load(k_at, t0 * BT, ks.n, tid);
    lv.load(v_at, t0 * BT, ks.n, tid);
  }
  for (int kt = t0; kt < t1; ++kt) {
    __syncthreads();
    lk.store(Ks, tid);
    lv.store(Vs, tid);
    __syncthreads();
    if (kt + 1 < t1) {
      lk.load(k_at, (kt + 1) * BT, ks.n, tid);
      lv.load(v_at, (kt + 1) * BT, ks.n, tid);
    }
    float ds[4][4];
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      Halves zh, dh;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        Frag<float> kf, vf;
        L::row(kf, Ks, jt * 16 + lr, 32 * s + 8 * lg);
        L::row(vf, Vs, jt * 16 + lr, 32 * s + 8 * lg);
        zh.add(s, kf, qf[s]);
        dh.add(s, vf, of[s]);
      }
      const f32x4_t z = zh.sum(), dp = dh.sum();
#pragma unroll
      for (int r = 0; r < 4; ++r)
        ds[jt][r] = kt * BT + jt * 16 + 4 * lg + r < ks.n ? exp_near(__builtin_fmaf(z[r], a.scale, -lse_i)) * (dp[r] - del) : 0.f;
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      Frag<float> df;
      frag_from_pair(df, ds, s2);
#pragma unroll
      for (int c = 0; c < NCT; ++c) {
        Frag<float> kf;
        L::col(kf, Ks, c * 16 + lr, s2, lg);
        mfma16(acc[c], kf, df);
      }
    }
  }
  float* row;
  float f = a.scale;
  if (a.splits > 1) {
    if (pi >= P) return;
    row = a.part + ((static_cast<int64_t>(it.split) * a.B * a.Hk + it.bh) * n_p + pi) * DH;
    f = 1.f;
  } else {
    if (pi >= (a.q_start ? P : n_p)) return;
    row = static_cast<float*>(a.dq) + at<DH>(a, qs, hk, pi, a.lddq);
  }
#pragma unroll
  for (int c = 0; c < NCT; ++c) {
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = pi < P ? acc[c][r] * f : 0.f;  // (padding: zeros)
    store_row4<float>(row + c * 16 + 4 * lg, v);
  }
}

// OWN_D: D of the range's queries is computed here into d_own (LDS).
template <int DH, bool OWN_D>
ATOM_DEV void dkdv_f32(float* Qs, float* Os, float* lse_s, float* del_s, float* d_own, const CrossArgs& a, int id) {
  using L = Tile<DH>;
  constexpr int NS = DH / 32, NCT = DH / 16;
  const Item it = item(a, id, a.k_x, a.k_splits);
  const Seq qs = seq(a.q_start, a.q_len, a.Tq, a.q_rows, it.b), ks = seq(a.k_start, a.k_len, a.Tk, a.k_rows, it.b);
  const int P = qs.n * a.G, k0 = it.x * 64, hk = it.hk;
  if (k0 >= ks.n && (a.k_splits > 1 || a.k_start)) return;
  const int64_t n_p = static_cast<int64_t>(a.Tq) * a.G;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lr = lane & 15, lg = lane >> 4;
  const int kj = k0 + w * 16 + lr;
  auto q_at = [&](int p) { return static_cast<const float*>(a.q) + at<DH>(a, qs, hk, p, a.ldq); };
  auto o_at = [&](int p) { return static_cast<const float*>(a.dout) + at<DH>(a, qs, hk, p, a.lddo); };

  Frag<float> kf[NS], vf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    frag_zero(kf[s]);
    frag_zero(vf[s]);
    if (kj < ks.n) {
      frag_load(kf[s], static_cast<const float*>(a.k) + (ks.row0 + kj) * a.ldk + hk * DH + 32 * s + 8 * lg);
      frag_load(vf[s], static_cast<const float*>(a.v) + (ks.row0 + kj) * a.ldv + hk * DH + 32 * s + 8 * lg);
    }
  }
  f32x4_t acc_k[NCT], acc_v[NCT];
#pragma unroll
  for (int c = 0; c < NCT; ++c) acc_k[c] = acc_v[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  int t0 = 0, t1 = 0;
  if (k0 < ks.n) range_of(P, a.k_splits, it.split, &t0, &t1);
  L lq, lo;
  float pre_lse = 0.f, pre_del = 0.f;
  auto fetch = [&](int t) {
    lq.load(q_at, t * BT, P, tid);
    lo.load(o_at, t * BT, P, tid);
    if (tid < BT) {
      const int i = t * BT + tid;
      pre_lse = INFINITY;
      pre_del = 0.f;
      if (i < P) {
        const Row rw = row_of(a, i);
        pre_lse = lse_of(a.lse[(qs.row0 + rw.t) * a.Hq + hk * a.G + rw.g]);
        if constexpr (!OWN_D) pre_del = a.delta[it.bh * n_p + i];
      }
    }
  };
  if (t0 < t1) fetch(t0);
  if constexpr (OWN_D) {  // (the loop's first barrier makes it visible)
    for (int r0 = t0 * BT; r0 < t1 * BT; r0 += 64) {
      const int r = r0 + w * 16 + lr;
      float v = 0.f;
      if (r < P) {
        const float* po = static_cast<const float*>(a.o) + at<DH>(a, qs, hk, r, a.ldo);
        const float* pd = o_at(r);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          Frag<float> f, g;
          frag_load(f, po + 32 * s + 8 * lg);
          frag_load(g, pd + 32 * s + 8 * lg);
          v += f.lo.x * g.lo.x + f.lo.y * g.lo.y + f.lo.z * g.lo.z + f.lo.w * g.lo.w;
          v += f.hi.x * g.hi.x + f.hi.y * g.hi.y + f.hi.z * g.hi.z + f.hi.w * g.hi.w;
        }
      }
      v = rows4_sum(v);
      if (lg == 0) d_own[r - t0 * BT] = v;
    }
  }
  for (int t = t0; t < t1; ++t) {
    __syncthreads();
    lq.store(Qs, tid);
    lo.store(Os, tid);
    if (tid < BT) lse_s[tid] = pre_lse, del_s[tid] = OWN_D ? d_own[(t - t0) * BT + tid] : pre_del;
    __syncthreads();
    if (t + 1 < t1) fetch(t + 1);
    float p[4][4], ds[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      Halves zh, dh;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        Frag<float> qf, of;
        L::row(qf, Qs, i * 16 + lr, 32 * s + 8 * lg);
        L::row(of, Os, i * 16 + lr, 32 * s + 8 * lg);
        zh.add(s, qf, kf[s]);
        dh.add(s, of, vf[s]);
      }
      const f32x4_t z = zh.sum(), dp = dh.sum();
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int il = i * 16 + 4 * lg + r;
        p[i][r] = exp_near(__builtin_fmaf(z[r], a.scale, -lse_s[il]));
        ds[i][r] = p[i][r] * (dp[r] - del_s[il]);
      }
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      Frag<float> pf, df;
      frag_from_pair(pf, p, s2);
      frag_from_pair(df, ds, s2);
#pragma unroll
      for (int c = 0; c < NCT; ++c) {
        Frag<float> of, qf;
        L::col(of, Os, c * 16 + lr, s2, lg);
        L::col(qf, Qs, c * 16 + lr, s2, lg);
        mfma16(acc_v[c], of, pf);
        mfma16(acc_k[c], qf, df);
      }
    }
  }
  float *rk, *rv;
  if (a.k_splits > 1) {
    if (kj >= ks.n) return;
    const int64_t r = (static_cast<int64_t>(it.split) * a.B * a.Hk + it.bh) * a.Tk + kj;
    rk = a.part_k + r * DH;
    rv = a.part_v + r * DH;
  } else {
    if (kj >= (a.k_start ? ks.n : a.Tk)) return;
    rk = static_cast<float*>(a.dk) + (ks.row0 + kj) * a.lddk + hk * DH;
    rv = static_cast<float*>(a.dv) + (ks.row0 + kj) * a.lddv + hk * DH;
  }
#pragma unroll
  for (int c = 0; c < NCT; ++c) {
    float vk[4], vv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      vk[i] = kj < ks.n ? acc_k[c][i] * a.scale : 0.f;  // (padding: zeros)
      vv[i] = kj < ks.n ? acc_v[c][i] : 0.f;
    }
    store_row4<float>(rk + c * 16 + 4 * lg, vk);
    store_row4<float>(rv + c * 16 + 4 * lg, vv);
  }
}

template <int DH>
__global__ void __launch_bounds__(256, 2) cross_dq_f32_kernel(const CrossArgs a) {
  __shared__ __attribute__((aligned(16))) float tiles[2][BT * Tile<DH>::RP];
  const int id = item_of(a.n_x * a.B * a.Hk * a.splits, blockIdx.x);
  if (id >= 0) dq_f32<DH>(tiles[0], tiles[1], a, id);
}
template <int DH>
__global__ void __launch_bounds__(256, 2) cross_dkdv_f32_kernel(const CrossArgs a) {
  __shared__ __attribute__((aligned(16))) float tiles[2][BT * Tile<DH>::RP];
  __shared__ float rows[2][BT];
  const int id = item_of(a.k_x * a.B * a.Hk * a.k_splits, blockIdx.x);
  if (id >= 0) dkdv_f32<DH, false>(tiles[0], tiles[1], rows[0], rows[1], nullptr, a, id);
}
// Small problems: both in one launch (see cross_bwd_small_kernel).
template <int DH>
__global__ void __launch_bounds__(256, 2) cross_bwd_small_f32_kernel(const CrossArgs a) {
  __shared__ __attribute__((aligned(16))) float tiles[2][BT * Tile<DH>::RP];
  __shared__ float rows[2][BT], d_own[SMALL_ROWS];
  const int n_k = a.dk ? a.k_x * a.B * a.Hk * a.k_splits : 0, n_q = a.dq ? a.n_x * a.B * a.Hk * a.splits : 0;
  const int k_end = (n_k + 7) & ~7, id = blockIdx.x;
  const int i = id < k_end ? item_of(n_k, id) : item_of(n_q, id - k_end);
  if (i < 0) return;
  if (id < k_end) dkdv_f32<DH, true>(tiles[0], tiles[1], rows[0], rows[1], d_own, a, i);
  else dq_f32<DH>(tiles[0], tiles[1], a, i);
}

}  // namespace cross

namespace {
unsigned grid_of(const CrossArgs& a, int64_t x, int64_t splits) {
  return static_cast<unsigned>((x * splits * a.B * a.Hk + 7) / 8 * 8);
}

template <int DH>
hipError_t bwd(const CrossArgs& a, bool small, hipStream_t s) {
  const unsigned nq = a.dq || a.delta ? grid_of(a, a.n_x, a.splits) : 0, nk = a.dk ? grid_of(a, a.k_x, a.k_splits) : 0;
  if (small) {
    if (nq + nk) hipLaunchKernelGGL(cross::cross_bwd_small_f32_kernel<DH>, dim3(nq + nk), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  if (nq) hipLaunchKernelGGL(cross::cross_dq_f32_kernel<DH>, dim3(nq), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !nk) return e;
  hipLaunchKernelGGL(cross::cross_dkdv_f32_kernel<DH>, dim3(nk), dim3(256), 0, s, a);
  return hipGetLastError();
}
}  // namespace

hipError_t cross_fwd_f32(const CrossArgs& a, int dh, hipStream_t s) {
  const dim3 grid(grid_of(a, a.n_x, a.splits));
  const bool few = static_cast<int64_t>(a.Tq) * a.G <= 16;
  if (dh == 64) {
    if (few) hipLaunchKernelGGL((cross::cross_fwd_f32_kernel<64, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cross::cross_fwd_f32_kernel<64, false>), grid, dim3(256), 0, s, a);
  } else {
    if (few) hipLaunchKernelGGL((cross::cross_fwd_f32_kernel<128, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cross::cross_fwd_f32_kernel<128, false>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}
hipError_t cross_bwd_f32(const CrossArgs& a, int dh, bool small, hipStream_t s) {
  return dh == 64 ? bwd<64>(a, small, s) : bwd<128>(a, small, s);
}

}  // namespace atom
