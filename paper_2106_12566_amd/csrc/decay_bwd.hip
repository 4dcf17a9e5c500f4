// Gradients of attention with a decaying bias (krpe_decay_bwd).  With the rows'
// G_i = [g_i | gd_i] = [dz_i | -(dz_i . z_i)] / den_i, A the state before a
// chunk and U the queries' sums phi(q_i) G_i^T after it:
//
//   dphi(q_i) = sum_{j <= i} e^{-rate (i - j)} (G_i . [v_j | 1]) phi(k_j) + e^{-rate (i + 1)} A^T G_i
//   dphi(k_j) = sum_{i >= j} e^{-rate (i - j)} (G_i . [v_j | 1]) phi(q_i) + e^{-rate (C - j)} U^T [v_j | 1]
//   dv_j      = sum_{i >= j} e^{-rate (i - j)} (phi(q_i) . phi(k_j)) g_i  + e^{-rate (C - j)} U phi(k_j)
//   dx        = W^T (dphi o phi) - x sum(dphi o phi)   (through the row's norm when normalising)
//
// (i, j in the chunk of C rows.)  One kernel has both sides: the queries'
// (SIDE 0) first sums its rows' numerators and denominators like the forward
// pass and leaves G behind for the sums backwards in time and for the keys'
// side (SIDE 1), whose first sums are dv.
//
// Bound by waits at one wave a SIMD in fp32 (204 registers, 150 KB of LDS) and two in bf16.  d = 64, n
// rows of a head and the terms' products counted: 24 heads, n = 4096, 128 features, fp32 (60 M d +
// 1920 (M + d) operations a row and side) 181 us a side, 0.47 PFLOP/s; 192 heads, n = 512, 64 features,
// bf16 (34 M d + 960 M + 800 d) 62 us, 0.40 PFLOP/s (a large bf16 product of the library 1.22).  Two
// work-groups a CU took bf16 from 79 us a side to 60; fp32 has no room for a second.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "decay.hpp"
#include "decay_states.hpp"

namespace krpe {

// 128 rows as operands over their columns: f[tile][ks][term][64], lane: row, column
// 16 ks + 8 (t / 4) + 4 lh + t % 4; zeros past the array's end and past d.
template <typename T, int DK>
struct RowTile {
  Raw4<T> u[DK][2];
  __device__ __forceinline__ void fetch(const Rows<T>& x) {
#pragma unroll
    for (int n = 0; n < DK; ++n) {
      const int e = threadIdx.x + 256 * n, r = e & 127, half = (e >> 7) & 1, ks = e >> 8;
      u[n][0].load(x, x.at(r), 16 * ks + 4 * half);
      u[n][1].load(x, x.at(r), 16 * ks + 4 * half + 8);
    }
  }
  template <int NT>
  __device__ __forceinline__ void put(uint4* __restrict__ f) const {
#pragma unroll
    for (int n = 0; n < DK; ++n) {
      const int e = threadIdx.x + 256 * n, r = e & 127, half = (e >> 7) & 1, ks = e >> 8;
      float v[4], w[4];
      u[n][0].values(v);
      u[n][1].values(w);
      uint32_t p[4][NT];
      split_pair<NT>(v[0], v[1], p[0]), split_pair<NT>(v[2], v[3], p[1]);
      split_pair<NT>(w[0], w[1], p[2]), split_pair<NT>(w[2], w[3], p[3]);
#pragma unroll
      for (int s = 0; s < NT; ++s)
        f[(((r >> 5) * DK + ks) * NT + s) * kFragLanes + 32 * half + (r & 31)] = make_uint4(p[0][s], p[1][s], p[2][s], p[3][s]);
    }
  }
};

// 32 rows of W from f0 turned: operands tl[ct][k2][term][64], lane: dimension, features in the
// slots (elu + 1: the identity).
template <int DT, int NT, bool ELU>
struct TurnedTile {
  static constexpr int N = (DT * 128 + 255) / 256;
  float v[N][8];
  __device__ __forceinline__ void fetch(const Rows<float>& W, int f0) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int e = threadIdx.x + 256 * n, c = e % (32 * DT), half = (e / (32 * DT)) & 1, k2 = e / (64 * DT);
      if (N * 256 > DT * 128 && e >= DT * 128) break;
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int l = f0 + 16 * k2 + 8 * (t >> 2) + 4 * half + (t & 3);
        if constexpr (ELU)
          v[n][t] = l == c ? 1.f : 0.f;
        else
          v[n][t] = W.one(W.at(W.at(l), c));
      }
    }
  }
  __device__ __forceinline__ void put(uint4* __restrict__ tl) const {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int e = threadIdx.x + 256 * n, c = e % (32 * DT), half = (e / (32 * DT)) & 1, k2 = e / (64 * DT);
      if (N * 256 > DT * 128 && e >= DT * 128) break;
      uint32_t q[4][NT];
#pragma unroll
      for (int j = 0; j < 4; ++j) split_pair<NT>(v[n][2 * j], v[n][2 * j + 1], q[j]);
#pragma unroll
      for (int s = 0; s < NT; ++s)
        tl[(((c >> 5) * 2 + k2) * NT + s) * kFragLanes + 32 * half + (c & 31)] = make_uint4(q[0][s], q[1][s], q[2][s], q[3][s]);
    }
  }
};

// Gradient of a lane's row (columns 32 t + 8 g + 4 lh + j along the registers) from
// y = W^T p (elu + 1: p itself) and sum(p).
template <typename TX, int DT, bool ELU>
__device__ __forceinline__ void store_row_gradient(const Rows<TX>& x, uint32_t at, floatx16 (&y)[DT], float sum,
                                                   TX* __restrict__ o, bool ok, bool nprf) {
  const int d = x.d;
  const int lh = (threadIdx.x & 63) >> 5;
  float xv[DT][16];
  float sq = 0.f;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float u[4];
      load4(x, at, 32 * t + 8 * g + 4 * lh, u);
#pragma unroll
      for (int j = 0; j < 4; ++j) xv[t][4 * g + j] = u[j], sq = fmaf(u[j], u[j], sq);
    }
  sq += __shfl_xor(sq, 32);
  const float inv = nprf ? (sq > 0.f ? rsqrtf(sq) : 0.f) : 1.f;
  float dot = 0.f;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      xv[t][e] *= inv;
      if constexpr (!ELU) y[t][e] = fmaf(-xv[t][e], sum, y[t][e]);
      dot = fmaf(xv[t][e], y[t][e], dot);
    }
  dot += __shfl_xor(dot, 32);
  if (!ok) return;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float u[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int e = 4 * g + j;
        u[j] = nprf ? fmaf(-xv[t][e], dot, y[t][e]) * inv : y[t][e];
      }
      store4(o, 32 * t + 8 * g + 4 * lh, d, u);
    }
}

// Terms of the other rows' values: v, exact in one where it is bf16, or g.
template <typename TX, int NT, int SIDE>
constexpr int kValueTerms = sizeof(TX) == 2 && SIDE == 0 ? 1 : NT;
// LDS in fragments: what the two passes and the step between work on; then the values' columns, there
// from the start, and after these R.  Where that is too much the columns come after the first pass,
// in its place.
template <typename TX, int DK, int NT, int SIDE>
struct GradSizes {
  static constexpr int NV = kValueTerms<TX, NT, SIDE>;
  static constexpr int kLoop = DK * 2 + 8 * NT + DK * NT + DK * NT, kRows = 4 * DK * NV;
  static constexpr int kWork = kLoop > kRows ? kLoop : kRows;
  static constexpr int kColumns = 4 * DK * NV, kR = 12 * NT;
  static constexpr bool kEarly = kWork + kColumns <= 152;
  static constexpr int kAll = kWork + (kEarly && kColumns > kR ? kColumns : kR);
};

template <typename TX, int DK, int NT, int SIDE, bool ELU>
__global__ __launch_bounds__(256, sizeof(TX) == 2 && DK <= 4 ? 2 : 1) void k_decay_grad(DecayArgs a) {
  using TG = typename std::conditional<SIDE == 0, TX, float>::type;  // values of the other rows: v, or g
  constexpr bool WHOLE = sizeof(TX) == 4;
  constexpr int NSX = kTermsX<TX>, DT = DK / 2, NW = 2;
  extern __shared__ __align__(16) uint4 smem[];
  constexpr int NV = kValueTerms<TX, NT, SIDE>, NG = kValueTerms<TX, NT, 1 - SIDE>;
  uint4* const wl = smem;                           // W [DK][NW][64]
  uint4* const kl = wl + DK * NW * kFragLanes;      // features of the other rows [4][2][NT][64]
  uint4* const sl = kl + 8 * NT * kFragLanes;       // the state [DT][2][NT][64], second pass [DK][NT][64]
  uint4* const tl = sl + DK * NT * kFragLanes;      // second pass: W turned [DT][2][NT][64]
  uint4* const vl = smem;                           // between: the values' rows [4][DK][NV][64]
  using Sizes = GradSizes<TX, DK, NT, SIDE>;
  uint4* const rl_ = smem + Sizes::kWork * kFragLanes;  // R off the diagonal [6][2][NT][64]
  uint4* const cl = Sizes::kEarly ? rl_ : smem;         // the values' columns [4][DT][2][NV][64]
  __shared__ __align__(16) float sden[32], sgd[kChunk], fr[kChunk], fc[kChunk];  // fr, fc: the other rows' factors
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int ch = blockIdx.x % a.nchunk, bh = blockIdx.x / a.nchunk, b = bh / a.H, h = bh % a.H, d = a.d;
  const int p0 = ch * kChunk, rows = rows_of(a.lens, b, a.n), cnt = min(kChunk, rows - p0);
  if (a.tail) {
    const size_t at = (static_cast<size_t>(bh) * a.n + p0) * d;
    clear_rows(static_cast<TX*>(SIDE == 0 ? a.dq : a.dk) + at, max(cnt, 0), min(kChunk, a.n - p0), d);
    if (SIDE == 1) clear_rows(static_cast<TX*>(a.dv) + at, max(cnt, 0), min(kChunk, a.n - p0), d);
  }
  if (cnt <= 0) return;
  const size_t base = static_cast<size_t>(bh) * a.n * d, cells = static_cast<size_t>(d + 1) * a.Mp;
  const float rl = rate_log2(a.rate[h]);
  const Rows<float> W(a.W + static_cast<size_t>(h) * a.M * d, a.M, d);
  const int seg = ch / a.segc, c0 = seg * a.segc, c1 = min(min(a.nchunk, c0 + a.segc), (rows + kChunk - 1) / kChunk);
  const bool inner = SIDE == 0 ? ch > c0 : ch + 1 < c1;
  const float* __restrict__ pre = inner ? (SIDE == 0 ? a.pre : a.preb) + (static_cast<size_t>(bh) * a.nchunk + ch) * cells : nullptr;
  const float* __restrict__ old =
      a.nseg > 1 ? (SIDE == 0 ? a.tot : a.totb) + (static_cast<size_t>(bh) * a.nseg + seg) * cells : nullptr;
  const float wold = decay(rl, SIDE == 0 ? (ch - c0) * kChunk : min(rows, c1 * kChunk) - (p0 + cnt));
  // the row tile of a wave: those with the most to do the other way round in every other 256
  // work-groups, which share a CU
  const int rt = (blockIdx.x >> 8) & 1 ? 3 - wave : wave;
  const int i = 32 * rt + lr;  // the lane's own row
  const float share = decay(rl, SIDE == 0 ? i + 1 : cnt - min(i, cnt));  // of the state outside the chunk
  const size_t from = base + static_cast<size_t>(p0) * d;
  const Rows<TX> own(static_cast<const TX*>(SIDE == 0 ? a.q : a.k) + from, cnt, d);
  const Rows<TX> oth(static_cast<const TX*>(SIDE == 0 ? a.k : a.q) + from, cnt, d);
  const Rows<TG> vals((SIDE == 0 ? static_cast<const TG*>(a.v) : reinterpret_cast<const TG*>(a.g)) + from, cnt, d);
  auto uses = [&](int t) { return SIDE == 0 ? t <= rt : t >= rt; };  // tiles of the other rows
  const TileWeights weights_of(rl, SIDE == 0 ? 1 : -1);
  auto weigh = [&](floatx16& x, int t) {
    if (t == rt)
      weights_of.template apply<true>(x, i, 32 * t);
    else
      weights_of.template apply<false>(x, i, 32 * t);
  };
  WeightTile<DK, NW, ELU, WHOLE> wt;
  wt.fetch(W, 0);
  StateTile<DT, NT, false> state(old, pre, wold, d, a.Mp);
  state.fetch(0);
  uint4 of[DK][NSX], tf[DK][NSX];
  RowFactors fo, ft;
  {
    Raw8<TX> x[DK], y[DK];
    fetch_row<TX, DK>(own, own.at(i), x);
    fetch_row<TX, DK>(oth, oth.at(i), y);
    if constexpr (Sizes::kEarly) stage_columns<TG, DT, 4, NV, Values::kAsIs>(vals, cl, nullptr);
    fo = row_factors<ELU, WHOLE>(row_square<TX, DK>(x), a.nprf, a.log2_m);
    ft = row_factors<ELU, WHOLE>(row_square<TX, DK>(y), a.nprf, a.log2_m);
#pragma unroll
    for (int ks = 0; ks < DK; ++ks) x[ks].terms(fo.x, of[ks]), y[ks].terms(ft.x, tf[ks]);
    if (lh == 0) fr[i] = ft.r, fc[i] = ft.c;
  }
  auto own_rows = [&](int ks, uint4(&x)[NSX]) {
#pragma unroll
    for (int n = 0; n < NSX; ++n) x[n] = of[ks][n];
  };
  auto other_rows = [&](int ks, uint4(&x)[NSX]) {
#pragma unroll
    for (int n = 0; n < NSX; ++n) x[n] = tf[ks][n];
  };
  auto weights = [&](int ks, uint4(&w)[NW]) { read_terms<NW>(wl + ks * NW * kFragLanes, w); };
  // [g | gd] of the lane's row (SIDE 0), or its values (SIDE 1)
  floatx16 G[DT];
  float gd = 1.f;
  RowTile<TG, DK> vrows;
  {
    floatx16 S[4], Z[DT];
#pragma unroll
    for (int t = 0; t < 4; ++t) S[t] = zero16();
#pragma unroll
    for (int t = 0; t < DT; ++t) Z[t] = zero16();
    float den = 0.f;
#pragma unroll 1
    for (int f0 = 0; f0 < a.Mp; f0 += 32) {
      // (the waves have all read the operands before: they have passed the barrier after phi)
      wt.put(wl);
      if (state.any()) state.put(sl, sden);
      if (f0 + 32 < a.Mp) {
        wt.fetch(W, f0 + 32);
        state.fetch(f0 + 32);
      }
      __syncthreads();
      floatx16 acc, lo, ph;
      const bool part = f0 + 32 > a.M;
      lo = zero16();
      project_terms<DK, NSX, NW, false, WHOLE>(weights, other_rows, acc, lo);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        ph[e] = feature<ELU, WHOLE>(acc[e], WHOLE ? lo[e] : 0.f, ft.r, ft.c);
        if (part && f0 + 8 * (e >> 2) + 4 * lh + (e & 3) >= a.M) ph[e] = 0.f;
      }
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        uint4 t[NT];
        pack_half<NT>(ph, k2, t);
#pragma unroll
        for (int s = 0; s < NT; ++s) kl[((rt * 2 + k2) * NT + s) * kFragLanes + lane] = t[s];
      }
      lo = zero16();
      project_terms<DK, NSX, NW, false, WHOLE>(weights, own_rows, acc, lo);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        ph[e] = feature<ELU, WHOLE>(acc[e], WHOLE ? lo[e] : 0.f, fo.r, fo.c);
        if (part && f0 + 8 * (e >> 2) + 4 * lh + (e & 3) >= a.M) ph[e] = 0.f;
      }
      uint4 po[2][NT];
      pack_half<NT>(ph, 0, po[0]);
      pack_half<NT>(ph, 1, po[1]);
      if (state.any()) {
        if constexpr (SIDE == 0) {
#pragma unroll
          for (int e = 0; e < 16; ++e) den = fmaf(sden[8 * (e >> 2) + 4 * lh + (e & 3)], ph[e], den);
        }
#pragma unroll
        for (int ct = 0; ct < DT; ++ct)
#pragma unroll
          for (int k2 = 0; k2 < 2; ++k2) {
            uint4 t[NT];
            read_terms<NT>(sl + (ct * 2 + k2) * NT * kFragLanes, t);
            Z[ct] = mfma_terms<NT, NT>(t, po[k2], Z[ct]);
          }
      }
      __syncthreads();
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (uses(t)) {
#pragma unroll
          for (int k2 = 0; k2 < 2; ++k2) {
            uint4 f[NT];
            read_terms<NT>(kl + (t * 2 + k2) * NT * kFragLanes, f);
            S[t] = mfma_terms<NT, NT>(f, po[k2], S[t]);
          }
        }
    }
    if constexpr (!Sizes::kEarly) {
      __syncthreads();
      stage_columns<TG, DT, 4, NV, Values::kAsIs>(vals, cl, nullptr);
      __syncthreads();
    }
    // (the next step's operands are asked for here)
    vrows.fetch(vals);
    const Rows<TX> mine(static_cast<const TX*>(SIDE == 0 ? a.dz : a.v) + from, cnt, d);
    Raw4<TX> m4[DT][4];
#pragma unroll
    for (int ct = 0; ct < DT; ++ct)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) m4[ct][g4].load(mine, mine.at(i), 32 * ct + 8 * g4 + 4 * lh);
    if (SIDE == 1 && threadIdx.x < kChunk)
      sgd[threadIdx.x] = static_cast<int>(threadIdx.x) < cnt ? a.gd[static_cast<size_t>(bh) * a.n + p0 + threadIdx.x] : 0.f;
    den *= share;
#pragma unroll
    for (int ct = 0; ct < DT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) Z[ct][e] *= share;
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (uses(t)) {
        weigh(S[t], t);
        if constexpr (SIDE == 0) {
#pragma unroll
          for (int e = 0; e < 16; ++e) den += S[t][e];
        }
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          uint4 pf[NT];
          pack_half<NT>(S[t], k2, pf);
#pragma unroll
          for (int ct = 0; ct < DT; ++ct) {
            uint4 f[NV];
            read_terms<NV>(cl + ((t * DT + ct) * 2 + k2) * NV * kFragLanes, f);
            Z[ct] = mfma_terms<NV, NT>(f, pf, Z[ct]);
          }
        }
      }
    if constexpr (SIDE == 0) {
      den += __shfl_xor(den, 32);
      const float inv = i < cnt ? 1.f / den : 0.f;
      float* __restrict__ g = a.g + from + static_cast<size_t>(i) * d;
      float dot = 0.f;
#pragma unroll
      for (int ct = 0; ct < DT; ++ct)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
          const int c = 32 * ct + 8 * g4 + 4 * lh;
          float u[4];
          m4[ct][g4].values(u);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            u[j] *= inv;
            dot = fmaf(u[j], Z[ct][4 * g4 + j], dot);
            G[ct][4 * g4 + j] = u[j];
          }
          if (i < cnt) store4(g, c, d, u);
        }
      gd = -(dot + __shfl_xor(dot, 32)) * inv;
      if (i < cnt && lh == 0) a.gd[static_cast<size_t>(bh) * a.n + p0 + i] = gd;
    } else {
      TX* __restrict__ dv = static_cast<TX*>(a.dv) + from + static_cast<size_t>(i) * d;
#pragma unroll
      for (int ct = 0; ct < DT; ++ct)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
          const int c = 32 * ct + 8 * g4 + 4 * lh;
          float u[4];
          m4[ct][g4].values(u);
#pragma unroll
          for (int j = 0; j < 4; ++j) G[ct][4 * g4 + j] = u[j];
          const float o[4] = {Z[ct][4 * g4], Z[ct][4 * g4 + 1], Z[ct][4 * g4 + 2], Z[ct][4 * g4 + 3]};
          if (i < cnt) store4(dv, c, d, o);
        }
    }
  }
  // R = e^{-rate (i - j)} (G_i . [v_j | 1]) as operands, and the lane's own values with the
  // weight of the state outside the chunk
  // (R of the diagonal tile stays in registers, of the others in LDS: each wave reads its own)
  uint4 R[2][NT], gf[DT][2][NT];
  auto r_at = [&](int t) { return rl_ + (SIDE == 0 ? rt * (rt - 1) / 2 + t : (3 - rt) * (2 - rt) / 2 + t - rt - 1) * 2 * NT * kFragLanes; };
  __syncthreads();  // the first pass's operands and the columns are consumed
  vrows.template put<NV>(vl);
  __syncthreads();
  uint4 ge[DT][2][NG];
#pragma unroll
  for (int ct = 0; ct < DT; ++ct)
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) pack_half<NG>(G[ct], k2, ge[ct][k2]);
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (uses(t)) {
      floatx16 r = zero16();
#pragma unroll
      for (int ks = 0; ks < DK; ++ks) {
        uint4 f[NV];
        read_terms<NV>(vl + (t * DK + ks) * NV * kFragLanes, f);
        r = mfma_terms<NV, NG>(f, ge[ks >> 1][ks & 1], r);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float one = SIDE == 0 ? gd : sgd[32 * t + 8 * (e >> 2) + 4 * lh + (e & 3)];
        r[e] += one;
      }
      weigh(r, t);
      if (t == rt) {
        pack_half<NT>(r, 0, R[0]);
        pack_half<NT>(r, 1, R[1]);
      } else {
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          uint4 f[NT];
          pack_half<NT>(r, k2, f);
#pragma unroll
          for (int s = 0; s < NT; ++s) r_at(t)[(k2 * NT + s) * kFragLanes + lane] = f[s];
        }
      }
    }
#pragma unroll
  for (int ct = 0; ct < DT; ++ct) {
#pragma unroll
    for (int e = 0; e < 16; ++e) G[ct][e] *= share;
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) pack_half<NT>(G[ct], k2, gf[ct][k2]);
  }
  const float one = gd * share;
  floatx16 Y[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) Y[t] = zero16();
  float psum = 0.f;
  // the state with rows l and the columns in the slots, and W with rows c and features in them
  StateTile<DT, NT, true> turned(old, pre, wold, d, a.Mp);
  TurnedTile<DT, NT, ELU> tt;
  wt.fetch(W, 0);
  turned.fetch(0);
  tt.fetch(W, 0);
#pragma unroll 1
  for (int f0 = 0; f0 < a.Mp; f0 += 32) {
    __syncthreads();  // the operands before consumed
    wt.put(wl);
    if (turned.any()) turned.put(sl, sden);
    tt.put(tl);
    if (f0 + 32 < a.Mp) {
      wt.fetch(W, f0 + 32);
      turned.fetch(f0 + 32);
      tt.fetch(W, f0 + 32);
    }
    __syncthreads();
    floatx16 acc, lo, ph, df = zero16();
    // features of the other rows, the positions along the registers
    lo = zero16();
    project_terms<DK, NSX, NW, true, WHOLE>(weights, other_rows, acc, lo);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 r4 = *reinterpret_cast<const float4*>(fr + 32 * rt + 8 * g + 4 * lh);
      const float4 c4 = *reinterpret_cast<const float4*>(fc + 32 * rt + 8 * g + 4 * lh);
      const float r_[4] = {r4.x, r4.y, r4.z, r4.w}, c_[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) ph[4 * g + j] = feature<ELU, WHOLE>(acc[4 * g + j], WHOLE ? lo[4 * g + j] : 0.f, r_[j], c_[j]);
    }
    if (f0 + lr >= a.M) ph = zero16();
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      uint4 t[NT];
      pack_half<NT>(ph, k2, t);
#pragma unroll
      for (int s = 0; s < NT; ++s) kl[((rt * 2 + k2) * NT + s) * kFragLanes + lane] = t[s];
    }
    if (turned.any()) {
#pragma unroll
      for (int ks = 0; ks < DK; ++ks) {
        uint4 f[NT];
        read_terms<NT>(sl + ks * NT * kFragLanes, f);
        df = mfma_terms<NT, NT>(f, gf[ks >> 1][ks & 1], df);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) df[e] = fmaf(sden[8 * (e >> 2) + 4 * lh + (e & 3)], one, df[e]);
    }
    lo = zero16();
    project_terms<DK, NSX, NW, false, WHOLE>(weights, own_rows, acc, lo);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int l = 8 * (e >> 2) + 4 * lh + (e & 3);
      ph[e] = feature<ELU, WHOLE>(acc[e], WHOLE ? lo[e] : 0.f, fo.r, fo.c);
      if constexpr (ELU) ph[e] = fminf(ph[e], 1.f);  // the slope of elu + 1 is e^x below zero, 1 above
      if (f0 + l >= a.M) ph[e] = 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (uses(t)) {
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          uint4 f[NT], y[NT];
          read_terms<NT>(kl + (t * 2 + k2) * NT * kFragLanes, f);
          if (t == rt) {
#pragma unroll
            for (int s = 0; s < NT; ++s) y[s] = R[k2][s];
          } else {
            read_terms<NT>(r_at(t) + k2 * NT * kFragLanes, y);
          }
          df = mfma_terms<NT, NT>(f, y, df);
        }
      }
#pragma unroll
    for (int e = 0; e < 16; ++e) ph[e] *= df[e], psum += ph[e];
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      uint4 pf[NT];
      pack_half<NT>(ph, k2, pf);
#pragma unroll
      for (int ct = 0; ct < DT; ++ct) {
        uint4 f[NT];
        read_terms<NT>(tl + (ct * 2 + k2) * NT * kFragLanes, f);
        Y[ct] = mfma_terms<NT, NT>(f, pf, Y[ct]);
      }
    }
  }
  psum += __shfl_xor(psum, 32);
  TX* __restrict__ out = static_cast<TX*>(SIDE == 0 ? a.dq : a.dk) + from + static_cast<size_t>(i) * d;
  store_row_gradient<TX, DT, ELU>(own, own.at(i), Y, psum, out, i < cnt, a.nprf);
}

namespace {

template <typename TX, int DK, bool ELU>
hipError_t go(const DecayArgs& a, hipStream_t st) {
  constexpr int NT = sizeof(TX) == 2 ? 2 : 3, NV = sizeof(TX) == 2 ? 1 : 3;
  constexpr int lds0 = GradSizes<TX, DK, NT, 0>::kAll * 1024, lds1 = GradSizes<TX, DK, NT, 1>::kAll * 1024;
  if constexpr (lds0 > 65536)
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&k_decay_grad<TX, DK, NT, 0, ELU>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, lds0);
  if constexpr (lds1 > 65536)
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&k_decay_grad<TX, DK, NT, 1, ELU>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, lds1);
  const dim3 grid(static_cast<unsigned>(a.B) * a.H * a.nchunk), block(256);
  const bool sums = a.nchunk > 1;  // (a single chunk has no state outside it)
  if (sums) launch_decay_states<TX, TX, DK, NT, NV, ELU, Sums::kForth>(a, st);
  hipLaunchKernelGGL((k_decay_grad<TX, DK, NT, 0, ELU>), grid, block, lds0, st, a);
  if (sums) launch_decay_states<TX, float, DK, NT, NT, ELU, Sums::kBack>(a, st);
  hipLaunchKernelGGL((k_decay_grad<TX, DK, NT, 1, ELU>), grid, block, lds1, st, a);
  return hipGetLastError();
}
template <typename TX, bool ELU>
hipError_t by_width(const DecayArgs& a, hipStream_t st) {
  if (a.d <= 32) return go<TX, 2, ELU>(a, st);
  if (a.d <= 64) return go<TX, 4, ELU>(a, st);
  if (a.d <= 96) return go<TX, 6, ELU>(a, st);
  return go<TX, 8, ELU>(a, st);
}

}  // namespace

hipError_t launch_decay_bwd(bool bf16, bool elu, const DecayArgs& a, hipStream_t st) {
  if (bf16) return elu ? by_width<uint16_t, true>(a, st) : by_width<uint16_t, false>(a, st);
  return elu ? by_width<float, true>(a, st) : by_width<float, false>(a, st);
}

}  // namespace krpe
