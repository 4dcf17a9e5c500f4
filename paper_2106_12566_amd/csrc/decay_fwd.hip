// Prompts of attention with a decaying bias (krpe_decay_fwd): the state's sums
// along each sequence, and the outputs of its chunks.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "decay.hpp"
#include "decay_states.hpp"

namespace krpe {

// Outputs of a chunk.  A wave owns 32 rows (lane: row i), per 32 features:
// its rows' phi(k) to LDS as fragments, phi(q) in registers; S^T[j][i] += phi(k)
// phi(q) for the row tiles j up to its own and the numerators' share of the
// state, A phi(q).  Then P = S e^{-rate (i - j)} leaves its registers as the
// operand of sum_j v_j P_ij.  W and the state of the next features are fetched
// while those at hand are worked on.
//
// Chunks of 128: the pairs inside (80 a row with the tiles left out) cost as much as a state of 80
// features.  Bound by waits: the row tiles' S and Z leave two waves a SIMD, which meet at two
// barriers for each 32 features.  d = 64, with the terms' products 24 M d + 960 (M + d) operations a row in
// fp32 and 12 M d + 160 M + 320 d in bf16: 96 heads, n = 4096, 128 features, fp32 256 us, 0.58 PFLOP/s;
// 16 heads, n = 16384, 256 features, bf16 122 us, 0.55 PFLOP/s (a large bf16 product of the library
// 1.22).  In the order of the waves (not turned in every other 256 work-groups) CUs with two last
// tiles on a SIMD end last.
// NT: terms of features and values; NP: of P and the state.
template <typename TX, int DK, int NT, int NP, bool ELU>
__device__ __forceinline__ void decay_out(const DecayArgs& a, int block) {
  constexpr bool WHOLE = sizeof(TX) == 4;
  constexpr int NSX = kTermsX<TX>, DT = DK / 2, NW = 2;
  constexpr bool KROWS = WHOLE;  // the rows of k through LDS, where registers are short
  extern __shared__ __align__(16) uint4 smem[];
  uint4* const wl = smem;                            // [DK][NW][64]
  uint4* const sl = wl + DK * NW * kFragLanes;       // [DT][2][NP][64]
  uint4* const kl = sl + DT * 2 * NP * kFragLanes;   // [4][2][NT][64]
  uint4* const xl = kl + 8 * NT * kFragLanes;        // KROWS: k [4][DK][NSX][64], each wave its own
  // the values' columns [4][DT][2][NT][64]: from the start, or after the features in their place
  constexpr bool EARLY = !KROWS;
  uint4* const vl = EARLY ? kl + 8 * NT * kFragLanes : smem;
  __shared__ __align__(16) float sden[32];
  __shared__ int odd;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int ch = block % a.nchunk, bh = block / a.nchunk, b = bh / a.H, h = bh % a.H, d = a.d;
  const int p0 = ch * kChunk, rows = rows_of(a.lens, b, a.n), cnt = min(kChunk, rows - p0);
  if (a.tail)
    clear_rows(static_cast<TX*>(a.z) + (static_cast<size_t>(bh) * a.n + p0) * d, max(cnt, 0), min(kChunk, a.n - p0), d);
  if (cnt <= 0) return;
  const int slot = a.state ? slot_of(a.slots, b, a.B, a.nslots) : kStateNone;
  const size_t base = static_cast<size_t>(bh) * a.n * d, cells = static_cast<size_t>(d + 1) * a.Mp;
  const float rl = rate_log2(a.rate[h]);
  const Rows<float> W(a.W + static_cast<size_t>(h) * a.M * d, a.M, d);
  const int seg = ch / a.segc, inseg = ch - seg * a.segc;
  const bool whole = a.nseg == 1;
  const float* __restrict__ pre =
      inseg || (whole && slot >= 0 && !a.fresh) ? a.pre + (static_cast<size_t>(bh) * a.nchunk + ch) * cells : nullptr;
  const float* __restrict__ old = whole ? nullptr : a.tot + (static_cast<size_t>(bh) * a.nseg + seg) * cells;
  StateTile<DT, NP, false> state(old, pre, decay(rl, inseg * kChunk), d, a.Mp);
  const bool has = state.any();
  // the row tile of a wave: the last ones have the most to do, so that every other 256 work-groups
  // (those that share a CU) have them the other way round
  const int rt = (block >> 8) & 1 ? 3 - wave : wave;
  const int i = 32 * rt + lr;
  const size_t from = base + static_cast<size_t>(p0) * d;
  const Rows<TX> qr(static_cast<const TX*>(a.q) + from, cnt, d), kr(static_cast<const TX*>(a.k) + from, cnt, d),
      vr(static_cast<const TX*>(a.v) + from, cnt, d);
  WeightTile<DK, NW, ELU, WHOLE> wt;
  wt.fetch(W, 0);
  state.fetch(0);
  uint4 qf[DK][NSX], kf[KROWS ? 1 : DK][NSX];
  RowFactors fq, fk;
  {
    Raw8<TX> x[DK], y[DK];
    fetch_row<TX, DK>(qr, qr.at(i), x);
    fetch_row<TX, DK>(kr, kr.at(i), y);
    if constexpr (EARLY) {
      if (threadIdx.x == 0) odd = 0;
      ColumnTile<TX, DT, 4, 256> t;
      t.fetch(vr, [&](int r) { return vr.at(r); });
      __syncthreads();  // (odd is clear)
      t.template put<NT, Values::kClean>(vl, &odd);
    }
    fq = row_factors<ELU, WHOLE>(row_square<TX, DK>(x), a.nprf, a.log2_m);
    fk = row_factors<ELU, WHOLE>(row_square<TX, DK>(y), a.nprf, a.log2_m);
#pragma unroll
    for (int ks = 0; ks < DK; ++ks) {
      x[ks].terms(fq.x, qf[ks]);
      if constexpr (KROWS) {
        uint4 t[NSX];
        y[ks].terms(fk.x, t);
#pragma unroll
        for (int n = 0; n < NSX; ++n) xl[((rt * DK + ks) * NSX + n) * kFragLanes + lane] = t[n];
      } else {
        y[ks].terms(fk.x, kf[ks]);
      }
    }
  }
  floatx16 S[4], Z[DT];
#pragma unroll
  for (int t = 0; t < 4; ++t) S[t] = zero16();
#pragma unroll
  for (int t = 0; t < DT; ++t) Z[t] = zero16();
  float den = 0.f;
  if (!EARLY && threadIdx.x == 0) odd = 0;
  auto weights = [&](int ks, uint4(&w)[NW]) { read_terms<NW>(wl + ks * NW * kFragLanes, w); };
#pragma unroll 1
  for (int f0 = 0; f0 < a.Mp; f0 += 32) {
    // (the waves have all read the operands before: they have passed the barrier after phi)
    wt.put(wl);
    if (has) state.put(sl, sden);
    if (f0 + 32 < a.Mp) {
      wt.fetch(W, f0 + 32);
      state.fetch(f0 + 32);
    }
    __syncthreads();
    floatx16 acc, lo, ph;
    const bool part = f0 + 32 > a.M;  // uniform: features past M weigh nothing
    auto features = [&](auto&& rows, const RowFactors& o) {
      lo = zero16();
      project_terms<DK, NSX, NW, false, WHOLE>(weights, rows, acc, lo);
#pragma unroll
      for (int e = 0; e < 16; ++e) ph[e] = feature<ELU, WHOLE>(acc[e], WHOLE ? lo[e] : 0.f, o.r, o.c);
      if (part) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (f0 + 8 * (e >> 2) + 4 * lh + (e & 3) >= a.M) ph[e] = 0.f;
      }
    };
    features(
        [&](int ks, uint4(&x)[NSX]) {
          if constexpr (KROWS) {
            read_terms<NSX>(xl + (rt * DK + ks) * NSX * kFragLanes, x);
          } else {
#pragma unroll
            for (int n = 0; n < NSX; ++n) x[n] = kf[ks][n];
          }
        },
        fk);
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      uint4 t[NT];
      pack_half<NT>(ph, k2, t);
#pragma unroll
      for (int s = 0; s < NT; ++s) kl[((rt * 2 + k2) * NT + s) * kFragLanes + lane] = t[s];
    }
    features(
        [&](int ks, uint4(&x)[NSX]) {
#pragma unroll
          for (int n = 0; n < NSX; ++n) x[n] = qf[ks][n];
        },
        fq);
    uint4 pq[2][NT];
    pack_half<NT>(ph, 0, pq[0]);
    pack_half<NT>(ph, 1, pq[1]);
    if (has) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 s4 = *reinterpret_cast<const float4*>(sden + 8 * g + 4 * lh);
        den = fmaf(s4.x, ph[4 * g], den), den = fmaf(s4.y, ph[4 * g + 1], den);
        den = fmaf(s4.z, ph[4 * g + 2], den), den = fmaf(s4.w, ph[4 * g + 3], den);
      }
#pragma unroll
      for (int ct = 0; ct < DT; ++ct)
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          uint4 t[NP];
          read_terms<NP>(sl + (ct * 2 + k2) * NP * kFragLanes, t);
          Z[ct] = mfma_terms<NP, NT>(t, pq[k2], Z[ct]);
        }
    }
    __syncthreads();  // phi(k) of all rows
#pragma unroll
    for (int jt = 0; jt < 4; ++jt)
      if (jt <= rt) {
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          uint4 t[NT];
          read_terms<NT>(kl + (jt * 2 + k2) * NT * kFragLanes, t);
          S[jt] = mfma_terms<NT, NT>(t, pq[k2], S[jt]);
        }
      }
  }
  // the state's share reaches row i over i + 1 positions
  const float since = decay(rl, i + 1);
  den *= since;
#pragma unroll
  for (int ct = 0; ct < DT; ++ct)
#pragma unroll
    for (int e = 0; e < 16; ++e) Z[ct][e] *= since;
  if constexpr (!EARLY) {
    __syncthreads();
    stage_columns<TX, DT, 4, NT, Values::kClean>(vr, vl, &odd);
  }
  const TileWeights weights_of(rl, 1);
  if constexpr (!EARLY) __syncthreads();
#pragma unroll
  for (int jt = 0; jt < 4; ++jt)
    if (jt <= rt) {
      if (jt == rt)
        weights_of.template apply<true>(S[jt], i, 32 * jt);
      else
        weights_of.template apply<false>(S[jt], i, 32 * jt);
#pragma unroll
      for (int e = 0; e < 16; ++e) den += S[jt][e];
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        uint4 pf[NP];
        pack_half<NP>(S[jt], k2, pf);
#pragma unroll
        for (int ct = 0; ct < DT; ++ct) {
          uint4 t[NT];
          read_terms<NT>(vl + ((jt * DT + ct) * 2 + k2) * NT * kFragLanes, t);
          Z[ct] = mfma_terms<NT, NP>(t, pf, Z[ct]);
        }
      }
    }
  den += __shfl_xor(den, 32);
  if (odd) {
    // values that are not finite (they went in as zeros): NaN for the rows that see them.
    // The same product over marks, 1 for such a value and 1 for a position that is seen.
    __syncthreads();
    stage_columns<TX, DT, 4, 1, Values::kMark>(vr, vl, nullptr);
    __syncthreads();
    for (int jt = 0; jt <= rt; ++jt)
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        floatx16 seen;
#pragma unroll
        for (int e = 0; e < 16; ++e) seen[e] = i >= 32 * jt + 8 * (e >> 2) + 4 * lh + (e & 3) ? 1.f : 0.f;
        uint4 pf[1];
        pack_half<1>(seen, k2, pf);
#pragma unroll
        for (int ct = 0; ct < DT; ++ct) {
          uint4 t[1];
          read_terms<1>(vl + ((jt * DT + ct) * 2 + k2) * kFragLanes, t);
          const floatx16 marks = mfma_bf16(t[0], pf[0], zero16());
#pragma unroll
          for (int e = 0; e < 16; ++e) Z[ct][e] = marks[e] > 0.f ? NAN : Z[ct][e];
        }
      }
  }
  if (i >= cnt) return;
  using TZ = TX;
  TZ* __restrict__ z = static_cast<TZ*>(a.z) + from + static_cast<size_t>(i) * d;
  const float inv = slot == kStateBad ? NAN : 1.f / den;
#pragma unroll
  for (int ct = 0; ct < DT; ++ct)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float o[4] = {Z[ct][4 * g] * inv, Z[ct][4 * g + 1] * inv, Z[ct][4 * g + 2] * inv, Z[ct][4 * g + 3] * inv};
      store4(z, 32 * ct + 8 * g + 4 * lh, d, o);
    }
}

template <typename TX, int DK, int NT, int NP, bool ELU>
__global__ __launch_bounds__(256, DK <= 4 ? 2 : 1) void k_decay_out(DecayArgs a) {
  decay_out<TX, DK, NT, NP, ELU>(a, blockIdx.x);
}

// Prompts of one chunk from empty states: their outputs need no sums, so that both are one launch, of
// as many work-groups for each head as there are groups of 128 features and one more.  One launch and
// two, n = 128, d = 64, us: 12 heads, bf16, 64 features 10.4 and 19.4; 128 heads 11.2 and 20.0; 192 heads
// (384 work-groups) 20.1 and 20.4; 256 features, 128 heads (384) 21.3 and 27.1, fp32 32.5 and 41.9; 192
// heads (576) 31.1 and 30.5, fp32 44.6 and 46.7; 256 heads (768) 38.7 and 31.4, fp32 56.5 and 47.9.
template <typename TX, int DK, int NT, int NP, bool ELU>
__global__ __launch_bounds__(256) void k_decay_short(DecayArgs a) {
  if (blockIdx.y == 0)
    decay_out<TX, DK, NT, NP, ELU>(a, blockIdx.x);
  else
    decay_states<TX, TX, DK, 3, NT, ELU, Sums::kForth, 4>(a, blockIdx.x, 0, blockIdx.y - 1);
}

namespace {

template <typename TX, int DK, bool ELU>
hipError_t go(const DecayArgs& a, hipStream_t st) {
  constexpr int NT = sizeof(TX) == 2 ? 1 : 3, NP = sizeof(TX) == 2 ? 2 : 3, DT = DK / 2;
  const int BH = a.B * a.H;
  constexpr int NSX = kTermsX<TX>, NW = 2;
  constexpr bool krows = sizeof(TX) == 4;  // (k_decay_out's KROWS)
  constexpr int feat = DK * NW + DT * 2 * NP + 8 * NT + (krows ? 4 * DK * NSX : 0), vals = 8 * DT * NT;
  constexpr int lds = (!krows ? feat + vals : feat > vals ? feat : vals) * 1024;
  if constexpr (lds > 65536)
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&k_decay_out<TX, DK, NT, NP, ELU>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  const bool one = a.nchunk == 1 && (!a.state || a.fresh);
  if constexpr (DK <= 4) {
    if (one && a.state && BH * (1 + (a.Mp / 32 + 3) / 4) <= 384) {
      if constexpr (lds + 49152 > 65536)
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&k_decay_short<TX, DK, NT, NP, ELU>),
                                  hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      hipLaunchKernelGGL((k_decay_short<TX, DK, NT, NP, ELU>), dim3(BH, 1 + (a.Mp / 32 + 3) / 4), dim3(256), lds, st, a);
      return hipGetLastError();
    }
  }
  // (a single chunk from zeros whose state is not kept needs no sums)
  if (a.state || !one) launch_decay_states<TX, TX, DK, 3, NT, ELU, Sums::kForth>(a, st);
  if (a.nchunk > 0)
    hipLaunchKernelGGL((k_decay_out<TX, DK, NT, NP, ELU>), dim3(static_cast<unsigned>(BH) * a.nchunk), dim3(256), lds, st, a);
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

hipError_t launch_decay_commit(bool bf16, bool elu, const DecayArgs& a, hipStream_t st) {
  auto go = [&](auto x, auto e) {
    using TX = decltype(x);
    constexpr int NV = sizeof(TX) == 2 ? 1 : 3;
    constexpr bool ELU = decltype(e)::value;
    if (a.d <= 32)
      launch_decay_states<TX, TX, 2, 3, NV, ELU, Sums::kPath>(a, st);
    else if (a.d <= 64)
      launch_decay_states<TX, TX, 4, 3, NV, ELU, Sums::kPath>(a, st);
    else if (a.d <= 96)
      launch_decay_states<TX, TX, 6, 3, NV, ELU, Sums::kPath>(a, st);
    else
      launch_decay_states<TX, TX, 8, 3, NV, ELU, Sums::kPath>(a, st);
  };
  if (bf16)
    elu ? go(uint16_t{}, std::true_type{}) : go(uint16_t{}, std::false_type{});
  else
    elu ? go(float{}, std::true_type{}) : go(float{}, std::false_type{});
  return hipGetLastError();
}

hipError_t launch_decay_fwd(bool bf16, bool elu, const DecayArgs& a, hipStream_t st) {
  if (bf16) return elu ? by_width<uint16_t, true>(a, st) : by_width<uint16_t, false>(a, st);
  return elu ? by_width<float, true>(a, st) : by_width<float, false>(a, st);
}

}  // namespace krpe
