// A tree of drafted tokens looked at from a sequence's state (krpe_decay_tree).
// Node t sees its ancestors and itself over the steps between their depths,
// and the state over depth(t) + 1 steps:
//
//   num_t | den_t = e^{-rate (dep_t + 1)} A phi(q_t)
//                 + sum_{a in anc(t)} e^{-rate (dep_t - dep_a)} (phi(q_t) . phi(k_a)) [v_a | 1]
//
// A work-group is one sequence and head, four waves: a row tile of 32 nodes or
// two, whose waves split the features.  What a wave needs of the state goes
// straight from memory into its operands, asked for before any row is worked
// on.  S = phi(K) phi(Q)^T and A phi(Q) leave the waves as partial sums, which
// are added through LDS in a fixed order.
//
// Bound by latency: the loads, the features, two sums through LDS.  64 x 16
// heads, 64 nodes, 256 features, d = 64 (100 MB in and out, 20 us at a plain
// copy's rate): 52 us, two work-groups on a CU, one of which loads while the
// other computes; with four waves for each of the two row tiles, one
// work-group on a CU, 69 us (a single sequence: 17.6 and 17.1 us).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "decay.hpp"

namespace krpe {

// kSplit: waves of a row tile; RT: row tiles (T <= 32 RT); NT: terms of features and values; NPP: of P and the state.
template <typename TX, int DK, int NT, int NPP, int RT, int kSplit, bool ELU>
__global__ __launch_bounds__(64 * kSplit * RT, sizeof(TX) == 2 && DK <= 4 ? 2 : 1) void k_decay_tree(PoolArgs a) {
  constexpr bool WHOLE = sizeof(TX) == 4;
  constexpr int THREADS = 64 * kSplit * RT, NX = sizeof(TX) / 2;
  constexpr int NSX = kTermsX<TX>, DT = DK / 2, NW = 2, NP = RT == 1 ? 1 : 3;
  constexpr int CG = DT % 2 ? 1 : 2;  // column tiles summed at a time
  // first the rows as they are [k, q][RT][DK][NX][64]; then the partial sums: S tiles [kSplit][NP], Z
  // [kSplit][RT][CG] a group of columns at a time
  constexpr int kRowsX = 2 * RT * DK * NX * 64, kTiles = NP > RT * CG ? NP : RT * CG, kPart = kSplit * kTiles * 16 * 16;
  __shared__ __align__(16) uint4 area[kRowsX > kPart ? kRowsX : kPart];
  uint4* const xl = area;
  float* const part = reinterpret_cast<float*>(area);
  __shared__ __align__(16) uint4 pl[NP][2][NPP][64];  // P as operands
  __shared__ __align__(16) uint4 vl[RT * DT * 2 * NT * 64];
  __shared__ float dpart[kSplit][32 * RT], dsum[NP][32];
  __shared__ float fr[2][32 * RT], fc[2][32 * RT], fx[2][32 * RT];
  __shared__ unsigned long long seen[32 * RT];
  __shared__ int odd;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 31, lh = lane >> 5, fw = wave % kSplit, r = wave / kSplit;
  const int b = blockIdx.x / a.H, h = blockIdx.x % a.H, d = a.d, T = a.T, M = a.M;
  const size_t base = static_cast<size_t>(blockIdx.x) * T * d;
  const Rows<TX> q(static_cast<const TX*>(a.q) + base, T, d), k(static_cast<const TX*>(a.k) + base, T, d),
      v(static_cast<const TX*>(a.v) + base, T, d);
  const Rows<float> W(a.W + static_cast<size_t>(h) * M * d, M, d);
  Raw8<TX> raw[DK];  // waves 0 .. 2 RT - 1: a row tile of k (even) or q
  const bool stages = wave < 2 * RT;
  if (stages) fetch_row<TX, DK>(wave & 1 ? q : k, v.at(32 * (wave >> 1) + lr), raw);
  ColumnTile<TX, DT, RT, THREADS> cols;
  cols.fetch(v, [&](int x) { return v.at(x); });
  float w8[DK][8];
  auto fetch_weights = [&](int f0) {
#pragma unroll
    for (int ks = 0; ks < DK; ++ks) load_weights<ELU>(W, f0 + lr, 16 * ks + 8 * lh, w8[ks]);
  };
  int slot = slot_in(a.slots, b, a.nslots);
  const float* __restrict__ st = slot >= 0 ? a.state + (static_cast<size_t>(slot) * a.H + h) * (d + 1) * M : nullptr;
  const Rows<float> sr(st ? st : a.state, st ? d + 1 : 0, M);  // (no state: zeros)
  const bool vec = M % 4 == 0;
  // (a column tile's share is asked for when the one before is used where registers are short)
  constexpr bool LATE = DK >= 6 || (WHOLE && DK == 4);
  float s8[LATE ? 1 : DT][2][8], sd[16];
  auto fetch_state = [&](int f0, int ct, float(&s)[2][8]) {
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      const int c = 32 * ct + lr, l = f0 + 16 * k2 + 4 * lh;
      const uint32_t o = sr.at(c);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if (vec) {
          const uint4 u = sr.b128(c < d && l + 8 * x < M ? o + 4u * (l + 8 * x) : kOut);
          s[k2][4 * x] = __uint_as_float(u.x), s[k2][4 * x + 1] = __uint_as_float(u.y);
          s[k2][4 * x + 2] = __uint_as_float(u.z), s[k2][4 * x + 3] = __uint_as_float(u.w);
        } else {
#pragma unroll
          for (int t = 0; t < 4; ++t)
            s[k2][4 * x + t] = sr.one(c < d && l + 8 * x + t < M ? o + 4u * (l + 8 * x + t) : kOut);
        }
      }
    }
  };
  auto fetch_last = [&](int f0) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int l = f0 + 8 * g + 4 * lh;
      if (vec) {
        const uint4 u = sr.b128(l < M ? sr.at(d) + 4u * l : kOut);
        sd[4 * g] = __uint_as_float(u.x), sd[4 * g + 1] = __uint_as_float(u.y);
        sd[4 * g + 2] = __uint_as_float(u.z), sd[4 * g + 3] = __uint_as_float(u.w);
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) sd[4 * g + t] = sr.one(l + t < M ? sr.at(d) + 4u * (l + t) : kOut);
      }
    }
  };
  const float rl = rate_log2(a.rate[h]);
  if (threadIdx.x == 0) odd = 0;
  if (wave == kSplit * RT - 1) {
    // ancestors by pointer doubling; a node without a valid parent, or below one, sees nothing
    int up = lane < T ? a.parent[static_cast<size_t>(b) * T + lane] : -2;
    bool dead = up < -1 || up >= lane;
    unsigned long long m = 1ull << lane;
    if (dead) up = -1;
    for (int s = 0; s < 6; ++s) {
      const int at = up < 0 ? lane : up;
      const unsigned lo = __shfl(static_cast<unsigned>(m), at), hi = __shfl(static_cast<unsigned>(m >> 32), at);
      const int dd = __shfl(static_cast<int>(dead), at), uu = __shfl(up, at);
      if (up >= 0) {
        m |= (static_cast<unsigned long long>(hi) << 32) | lo;
        dead |= dd != 0;
        up = uu;
      }
    }
    if (lane < 32 * RT) seen[lane] = dead ? 0ull : m;
  }
  floatx16 S[RT], Z[DT];  // S: (key tile 0 and, in row tile 1, key tile 1)
  float den = 0.f;
#pragma unroll
  for (int t = 0; t < RT; ++t) S[t] = zero16();
#pragma unroll
  for (int t = 0; t < DT; ++t) Z[t] = zero16();
  int f0 = 32 * fw;
#pragma unroll 1
  do {  // (a wave without features has zeros)
    fetch_weights(f0);
    if constexpr (!LATE) {
#pragma unroll
      for (int ct = 0; ct < DT; ++ct) fetch_state(f0, ct, s8[ct]);
    }
    fetch_last(f0);
    if (f0 < 32 * kSplit) {  // the first time
      if (stages) {
        const RowFactors o = row_factors<ELU, WHOLE>(row_square<TX, DK>(raw), a.nprf, a.log2_m);
        const int w = wave & 1, t = wave >> 1;
        if (lh == 0) fr[w][32 * t + lr] = o.r, fc[w][32 * t + lr] = o.c, fx[w][32 * t + lr] = o.x;
#pragma unroll
        for (int ks = 0; ks < DK; ++ks)
#pragma unroll
          for (int n = 0; n < NX; ++n) xl[(((w * RT + t) * DK + ks) * NX + n) * 64 + lane] = raw[ks].u[n];
      }
      __syncthreads();  // (odd is clear)
      cols.template put<NT, Values::kClean>(vl, &odd);
    }
    uint4 wf[DK][NW];
#pragma unroll
    for (int ks = 0; ks < DK; ++ks) weight_terms<NW, WHOLE>(w8[ks], wf[ks]);
    // features of a row tile (lane: row; features along the registers), zeros past M
    auto features = [&](int w, int t, floatx16& ph, uint4(&p)[2][NT]) {
      const float scale = fx[w][32 * t + lr];
      floatx16 acc, lo = zero16();
      project_terms<DK, NSX, NW, false, WHOLE>(
          [&](int ks, uint4(&y)[NW]) {
#pragma unroll
            for (int n = 0; n < NW; ++n) y[n] = wf[ks][n];
          },
          [&](int ks, uint4(&y)[NSX]) {
            Raw8<TX> x;
            read_terms<NX>(xl + ((w * RT + t) * DK + ks) * NX * 64, x.u);
            x.terms(scale, y);
          },
          acc, lo);
      const float r_ = fr[w][32 * t + lr], c_ = fc[w][32 * t + lr];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        ph[e] = feature<ELU, WHOLE>(acc[e], WHOLE ? lo[e] : 0.f, r_, c_);
        if (f0 + 8 * (e >> 2) + 4 * lh + (e & 3) >= M) ph[e] = 0.f;
      }
      pack_half<NT>(ph, 0, p[0]);
      pack_half<NT>(ph, 1, p[1]);
    };
    uint4 pk[2][NT], pq[2][NT];
    floatx16 ph;
    features(1, r, ph, pq);
#pragma unroll
    for (int e = 0; e < 16; ++e) den = fmaf(ph[e], sd[e], den);
#pragma unroll
    for (int ct = 0; ct < DT; ++ct) {
      if constexpr (LATE) fetch_state(f0, ct, s8[0]);
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        const float(&x)[8] = s8[LATE ? 0 : ct][k2];
        uint32_t p[4][NPP];
#pragma unroll
        for (int j = 0; j < 4; ++j) split_pair<NPP>(x[2 * j], x[2 * j + 1], p[j]);
        uint4 t[NPP];
#pragma unroll
        for (int s = 0; s < NPP; ++s) t[s] = make_uint4(p[0][s], p[1][s], p[2][s], p[3][s]);
        Z[ct] = mfma_terms<NPP, NT>(t, pq[k2], Z[ct]);
      }
    }
    features(0, 0, ph, pk);
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) S[0] = mfma_terms<NT, NT>(pk[k2], pq[k2], S[0]);
    if (RT == 2 && r == 1) {
      features(0, 1, ph, pk);
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) S[RT - 1] = mfma_terms<NT, NT>(pk[k2], pq[k2], S[RT - 1]);
    }
    f0 += 32 * kSplit;
  } while (f0 < M);
  __syncthreads();  // the rows are consumed: their place takes the sums
  // S, tile t: (row tile, key tile) = (0, 0), (1, 0), (1, 1): the waves' sums, masked and weighted, as
  // operands
  auto put = [&](int t, int tiles, const floatx16& x) {
#pragma unroll
    for (int e = 0; e < 16; ++e) part[((fw * tiles + t) * 16 + e) * 64 + lane] = x[e];
  };
  put(r, NP, S[0]);
  if (RT == 2 && r == 1) put(2 % NP, NP, S[RT - 1]);
  den += __shfl_xor(den, 32);
  if (lh == 0) dpart[fw][32 * r + lr] = den;
  __syncthreads();
  if (wave < NP) {
    const int t = wave, it = t ? 1 : 0, jt = t == 2 ? 1 : 0;
    const int i = 32 * it + lr;
    const unsigned long long m = seen[i];
    const int dep = __popcll(m) - 1;
    floatx16 p;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int j = 32 * jt + 8 * (e >> 2) + 4 * lh + (e & 3);
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < kSplit; ++w) x += part[((w * NP + t) * 16 + e) * 64 + lane];
      p[e] = (m >> j) & 1 ? x * decay(rl, dep - (__popcll(seen[j]) - 1)) : 0.f;
      s += p[e];
    }
    s += __shfl_xor(s, 32);
    if (lh == 0) dsum[t][lr] = s;
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      uint4 f[NPP];
      pack_half<NPP>(p, k2, f);
#pragma unroll
      for (int n = 0; n < NPP; ++n) pl[t][k2][n][lane] = f[n];
    }
  }
  slot = check_slot(a.slots, slot, b, a.B);
  TX* __restrict__ z = static_cast<TX*>(a.z) + base;
  const int i = 32 * r + lr;
  const unsigned long long m = seen[i];
  const float since = decay(rl, __popcll(m));
  float inv = 0.f;
#pragma unroll
  for (int g = 0; g < DT / CG; ++g) {
    __syncthreads();
#pragma unroll
    for (int ct = 0; ct < CG; ++ct) put(r * CG + ct, RT * CG, Z[CG * g + ct]);
    __syncthreads();
    if (g == 0) {
      float dn = 0.f;
#pragma unroll
      for (int w = 0; w < kSplit; ++w) dn += dpart[w][i];
      dn = dn * since + (r ? dsum[1 % NP][lr] + dsum[2 % NP][lr] : dsum[0][lr]);
      inv = slot == kStateBad ? NAN : (m ? 1.f / dn : 0.f);
    }
    if (fw < CG) {
      const int ct = CG * g + fw;
      floatx16 o;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kSplit; ++w) x += part[((w * RT * CG + r * CG + fw) * 16 + e) * 64 + lane];
        o[e] = m ? x * since : 0.f;  // (no NaN of the state where nothing is seen)
      }
#pragma unroll
      for (int jt = 0; jt < RT; ++jt)
        if (jt <= r) {
#pragma unroll
          for (int k2 = 0; k2 < 2; ++k2) {
            uint4 vf[NT], pf[NPP];
            read_terms<NT>(vl + ((jt * DT + ct) * 2 + k2) * NT * 64, vf);
            read_terms<NPP>(&pl[r + jt][k2][0][0], pf);
            o = mfma_terms<NT, NPP>(vf, pf, o);
          }
        }
      if (odd) {
        // values that are not finite went in as zeros: NaN for the nodes that see them
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int c = 32 * ct + 8 * (e >> 2) + 4 * lh + (e & 3);
          if (c < d)
            for (int j = 0; j < T; ++j)
              if (((m >> j) & 1) && !finite(v.one(v.at(v.at(j), c)))) o[e] = NAN;
        }
      }
      if (i < T) {
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const float o4[4] = {o[4 * e4] * inv, o[4 * e4 + 1] * inv, o[4 * e4 + 2] * inv, o[4 * e4 + 3] * inv};
          store4(z + static_cast<size_t>(i) * d, 32 * ct + 8 * e4 + 4 * lh, d, o4);
        }
      }
    }
  }
}

namespace {
template <typename TX, int DK, bool ELU>
hipError_t go(const PoolArgs& a, hipStream_t st) {
  constexpr int NT = sizeof(TX) == 2 ? 1 : 3, NP = sizeof(TX) == 2 ? 2 : 3;
  const dim3 grid(static_cast<unsigned>(a.B) * a.H);
  if (a.T <= 32)
    hipLaunchKernelGGL((k_decay_tree<TX, DK, NT, NP, 1, 4, ELU>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_decay_tree<TX, DK, NT, NP, 2, 2, ELU>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}
template <typename TX, bool ELU>
hipError_t by_width(const PoolArgs& a, hipStream_t st) {
  if (a.d <= 32) return go<TX, 2, ELU>(a, st);
  if (a.d <= 64) return go<TX, 4, ELU>(a, st);
  if (a.d <= 96) return go<TX, 6, ELU>(a, st);
  return go<TX, 8, ELU>(a, st);
}
}  // namespace

hipError_t launch_decay_tree(bool bf16, bool elu, const PoolArgs& a, hipStream_t st) {
  if (bf16) return elu ? by_width<uint16_t, true>(a, st) : by_width<uint16_t, false>(a, st);
  return elu ? by_width<float, true>(a, st) : by_width<float, false>(a, st);
}

}  // namespace krpe
