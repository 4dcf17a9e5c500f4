// A tree of drafted tokens looked at from a sequence's state (krpe_decay_tree).
// Node t sees its ancestors and itself over the steps between their depths,
// and the state over depth(t) + 1 steps:
//
//   num_t | den_t = e^{-rate (dep_t + 1)} A phi(q_t)
//                 + sum_{a in anc(t)} e^{-rate (dep_t - dep_a)} (phi(q_t) . phi(k_a)) [v_a | 1]
//
// A work-group is one sequence and head.  Its waves split the features (the
// state is read once, straight into operands, by the wave whose features they
// are), so S = phi(K) phi(Q)^T and A phi(Q) leave the waves as partial sums,
// which are added through LDS in a fixed order.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "decay.hpp"

namespace krpe {

constexpr int kTreeWaves = 4;

// RT: row tiles of 32 nodes (T <= 32 RT); NT: terms of features and values; NPP: of P and the state.
template <typename TX, int DK, int NT, int NPP, int RT, bool ELU>
__global__ __launch_bounds__(64 * kTreeWaves) void k_decay_tree(PoolArgs a) {
  constexpr bool WHOLE = sizeof(TX) == 4;
  constexpr int NSX = kTermsX<TX>, DT = DK / 2, NW = WHOLE ? 3 : 2, NP = RT == 1 ? 1 : 3;
  // partial sums: S tiles [wave][NP], then one row tile's Z [wave][DT] at a time
  constexpr int kPart = kTreeWaves * (NP > DT ? NP : DT) * 16;
  __shared__ __align__(16) float part[kPart * 64];
  __shared__ __align__(16) uint4 pl[NP][2][NPP][64];      // P as operands
  __shared__ __align__(16) uint4 vl[RT * DT * 2 * NT * 64];
  __shared__ float dpart[kTreeWaves][32 * RT], dsum[NP][32];
  __shared__ unsigned long long seen[32 * RT];
  __shared__ int odd;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int b = blockIdx.x / a.H, h = blockIdx.x % a.H, d = a.d, T = a.T, M = a.M;
  const int slot = slot_of(a.slots, b, a.B, a.nslots);
  const float* __restrict__ st = slot >= 0 ? a.state + (static_cast<size_t>(slot) * a.H + h) * (d + 1) * M : nullptr;
  const size_t base = static_cast<size_t>(blockIdx.x) * T * d;
  const Rows<TX> q(static_cast<const TX*>(a.q) + base, T, d), k(static_cast<const TX*>(a.k) + base, T, d),
      v(static_cast<const TX*>(a.v) + base, T, d);
  const Rows<float> W(a.W + static_cast<size_t>(h) * M * d, M, d);
  const float rl = rate_log2(a.rate[h]);
  if (threadIdx.x == 0) odd = 0;
  if (wave == 0) {
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
  __syncthreads();
  stage_columns<TX, DT, RT, NT, Values::kClean>(v, vl, &odd);
  floatx16 S[NP], Z[RT][DT];
  float den[RT];
#pragma unroll
  for (int t = 0; t < NP; ++t) S[t] = zero16();
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    den[r] = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) Z[r][t] = zero16();
  }
  const bool vec = M % 4 == 0;
  for (int f0 = 32 * wave; f0 < M; f0 += 32 * kTreeWaves) {
    uint4 wf[DK][NW];
#pragma unroll
    for (int ks = 0; ks < DK; ++ks) {
      float v8[8];
      load_weights<ELU>(W, f0 + lr, 16 * ks + 8 * lh, v8);
      uint4 t3[3];
      split_bf16x8(v8, t3);
#pragma unroll
      for (int s = 0; s < NW; ++s) wf[ks][s] = t3[s];
    }
    // features of a row tile (lane: row; features along the registers), zeros past M
    auto features = [&](const Rows<TX>& x, int r, floatx16& ph) {
      const int i = 32 * r + lr;
      Raw8<TX> raw[DK];
      fetch_row<TX, DK>(x, x.at(i), raw);
      const RowFactors o = row_factors<ELU>(row_square<TX, DK>(raw), a.nprf, a.log2_m);
      uint4 xf[DK][NSX];
#pragma unroll
      for (int ks = 0; ks < DK; ++ks) raw[ks].terms(xf[ks]);
      floatx16 acc, lo;
      project_terms<DK, NSX, NW, false, WHOLE>(
          [&](int ks, uint4(&w)[NW]) {
#pragma unroll
            for (int n = 0; n < NW; ++n) w[n] = wf[ks][n];
          },
          xf, acc, lo);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        ph[e] = feature<ELU, WHOLE>(acc[e], WHOLE ? lo[e] : 0.f, o.r, o.c, o.f);
        if (f0 + 8 * (e >> 2) + 4 * lh + (e & 3) >= M) ph[e] = 0.f;
      }
    };
    uint4 pk[RT][2][NT], pq[RT][2][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      floatx16 ph;
      features(k, r, ph);
      pack_half<NT>(ph, 0, pk[r][0]);
      pack_half<NT>(ph, 1, pk[r][1]);
      features(q, r, ph);
      pack_half<NT>(ph, 0, pq[r][0]);
      pack_half<NT>(ph, 1, pq[r][1]);
      if (st) {
        const float* __restrict__ sd = st + static_cast<size_t>(d) * M;
#pragma unroll
        for (int e = 0; e < 16; ++e) den[r] = fmaf(ph[e], sd[min(f0 + 8 * (e >> 2) + 4 * lh + (e & 3), M - 1)], den[r]);
      }
    }
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      S[0] = mfma_terms<NT, NT>(pk[0][k2], pq[0][k2], S[0]);
      if constexpr (RT == 2) {
        S[1] = mfma_terms<NT, NT>(pk[0][k2], pq[1][k2], S[1]);
        S[2] = mfma_terms<NT, NT>(pk[1][k2], pq[1][k2], S[2]);
      }
    }
    if (st) {
#pragma unroll
      for (int ct = 0; ct < DT; ++ct) {
        const int c = 32 * ct + lr;
        const float* __restrict__ sr = st + static_cast<size_t>(min(c, d)) * M;
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          floatx16 x = zero16();  // (eight used)
          const int l = f0 + 16 * k2 + 4 * lh;
          if (c < d) {
            if (vec && l + 12 <= M) {
              const float4 u = *reinterpret_cast<const float4*>(sr + l), w = *reinterpret_cast<const float4*>(sr + l + 8);
              x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = w.x, x[5] = w.y, x[6] = w.z, x[7] = w.w;
            } else {
#pragma unroll
              for (int t = 0; t < 8; ++t) {
                const int at = l + (t & 3) + 8 * (t >> 2);
                x[t] = at < M ? sr[at] : 0.f;
              }
            }
          }
          uint4 t[NPP];
          pack_half<NPP>(x, 0, t);
#pragma unroll
          for (int r = 0; r < RT; ++r) Z[r][ct] = mfma_terms<NPP, NT>(t, pq[r][k2], Z[r][ct]);
        }
      }
    }
  }
  // S: the waves' sums, masked and weighted, as operands
#pragma unroll
  for (int t = 0; t < NP; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) part[((wave * NP + t) * 16 + e) * 64 + lane] = S[t][e];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float s = den[r] + __shfl_xor(den[r], 32);
    if (lh == 0) dpart[wave][32 * r + lr] = s;
  }
  __syncthreads();
  for (int t = wave; t < NP; t += kTreeWaves) {
    const int it = t ? 1 : 0, jt = t == 2 ? 1 : 0;  // (row tile, column tile)
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
      for (int w = 0; w < kTreeWaves; ++w) x += part[((w * NP + t) * 16 + e) * 64 + lane];
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
  TX* __restrict__ z = static_cast<TX*>(a.z) + base;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    __syncthreads();
#pragma unroll
    for (int ct = 0; ct < DT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) part[((wave * DT + ct) * 16 + e) * 64 + lane] = Z[r][ct][e];
    __syncthreads();
    const int i = 32 * r + lr;
    const unsigned long long m = seen[i];
    const float since = decay(rl, __popcll(m));
    float dn = 0.f;
#pragma unroll
    for (int w = 0; w < kTreeWaves; ++w) dn += dpart[w][i];
    dn = dn * since + (r ? dsum[1][lr] + dsum[2 % NP][lr] : dsum[0][lr]);
    const float inv = slot == kStateBad ? NAN : (m ? 1.f / dn : 0.f);
    for (int ct = wave; ct < DT; ct += kTreeWaves) {
      floatx16 o;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kTreeWaves; ++w) x += part[((w * DT + ct) * 16 + e) * 64 + lane];
        o[e] = m ? x * since : 0.f;  // (no NaN of the state where nothing is seen)
      }
#pragma unroll
      for (int jt = 0; jt <= r; ++jt)
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          uint4 vf[NT], pf[NPP];
          read_terms<NT>(vl + ((jt * DT + ct) * 2 + k2) * NT * 64, vf);
          read_terms<NPP>(&pl[r + jt][k2][0][0], pf);
          o = mfma_terms<NT, NPP>(vf, pf, o);
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
      if (i < T)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float o4[4] = {o[4 * g] * inv, o[4 * g + 1] * inv, o[4 * g + 2] * inv, o[4 * g + 3] * inv};
          store4(z + static_cast<size_t>(i) * d, 32 * ct + 8 * g + 4 * lh, d, o4);
        }
    }
  }
}

namespace {
template <typename TX, int DK, bool ELU>
hipError_t go(const PoolArgs& a, hipStream_t st) {
  constexpr int NT = sizeof(TX) == 2 ? 1 : 3, NP = sizeof(TX) == 2 ? 2 : 3;
  const dim3 grid(static_cast<unsigned>(a.B) * a.H), block(64 * kTreeWaves);
  if (a.T <= 32)
    hipLaunchKernelGGL((k_decay_tree<TX, DK, NT, NP, 1, ELU>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((k_decay_tree<TX, DK, NT, NP, 2, ELU>), grid, block, 0, st, a);
  return hipGetLastError();
}
template <typename TX, bool ELU>
hipError_t by_width(const PoolArgs& a, hipStream_t st) {
  if (a.d <= 32) return go<TX, 2, ELU>(a, st);
  if (a.d <= 64) return go<TX, 4, ELU>(a, st);
  return go<TX, 8, ELU>(a, st);
}
}  // namespace

hipError_t launch_decay_tree(bool bf16, bool elu, const PoolArgs& a, hipStream_t st) {
  if (bf16) return elu ? by_width<uint16_t, true>(a, st) : by_width<uint16_t, false>(a, st);
  return elu ? by_width<float, true>(a, st) : by_width<float, false>(a, st);
}

}  // namespace krpe
