// The sums of a decaying state along a sequence, forwards (the keys' [v | 1]) and
// backwards in time (the queries' gradients): by chunk within segments, then
// joined over the segments.  Used by the prompts and by the gradients.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "decay.hpp"

namespace krpe {

// Sums of a segment's chunks: pre[chunk] = the segment's state before the chunk,
// tot[segment] = the one behind its last.  A wave owns 32 features, its sums
// in registers (lane: feature; value columns along the registers), and its W;
// the rows of x and v pass through LDS for all waves of the work-group.
//
// With REV the queries' sums backwards in time, of phi(q_i) [g_i | gd_i]: the rows' weights go
// to the chunk's first position, and "before" is after.
template <typename TX, typename TV, int DK, int NP, int NV, bool ELU, bool REV>
__global__ __launch_bounds__(256) void k_decay_states(DecayArgs a) {
  constexpr int NSX = kTermsX<TX>, DT = DK / 2;
  constexpr int PB = NSX == 3 && DK == 8 ? 2 : 4;  // 32-row blocks staged at a time
  extern __shared__ __align__(16) uint4 smem[];
  uint4* const xl = smem;                               // [PB][DK][NSX][64]
  uint4* const vl = xl + PB * DK * NSX * kFragLanes;    // [PB][DT][2][NV][64]
  __shared__ __align__(16) float fr[32 * PB], fc[32 * PB], ff[32 * PB], fd[REV ? 32 * PB : 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6, lr = lane & 31, lh = lane >> 5;
  const int seg = blockIdx.y, fg = blockIdx.z, bh = blockIdx.x, h = bh % a.H, d = a.d;
  const int l = (fg * waves + wave) * 32 + lr;
  const size_t cells = static_cast<size_t>(d + 1) * a.Mp;
  const TX* __restrict__ k = static_cast<const TX*>(REV ? a.q : a.k) + static_cast<size_t>(bh) * a.n * d;
  const TV* __restrict__ v = static_cast<const TV*>(REV ? a.g : a.v) + static_cast<size_t>(bh) * a.n * d;
  float* const pre = REV ? a.preb : a.pre;
  const float rl = rate_log2(a.rate[h]);
  const int rows = rows_of(a.lens, bh / a.H, a.n);
  uint4 wf[DK][3];
#pragma unroll
  for (int ks = 0; ks < DK; ++ks) {
    const int c = 16 * ks + 8 * lh;
    float v8[8];
    if constexpr (ELU) {
#pragma unroll
      for (int t = 0; t < 8; ++t) v8[t] = c + t == l ? 1.f : 0.f;
    } else {
      load8(a.W + (static_cast<size_t>(h) * a.M + min(l, a.M - 1)) * d + min(c, d - 1), l < a.M ? d - c : 0, d % 4 == 0,
            v8);
    }
    split_bf16x8(v8, wf[ks]);
  }
  floatx16 S[DT];
#pragma unroll
  for (int ct = 0; ct < DT; ++ct) S[ct] = zero16();
  float sum = 0.f;  // of this lane half's positions
  auto store = [&](float* __restrict__ to) {
    if (l >= a.Mp) return;
#pragma unroll
    for (int ct = 0; ct < DT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int c = 32 * ct + 8 * (e >> 2) + 4 * lh + (e & 3);
        if (c < d) to[static_cast<size_t>(c) * a.Mp + l] = S[ct][e];
      }
    const float s = sum + __shfl_xor(sum, 32);
    if (lh == 0) to[static_cast<size_t>(d) * a.Mp + l] = s;
  };
  const int c0 = seg * a.segc, c1 = min(min(a.nchunk, c0 + a.segc), (rows + kChunk - 1) / kChunk);
  for (int s = c0; s < c1; ++s) {
    const int ch = REV ? c0 + c1 - 1 - s : s;
    const int p0 = ch * kChunk, cnt = min(kChunk, rows - p0);
    if (s != c0) {
      store(pre + (static_cast<size_t>(bh) * a.nchunk + ch) * cells);
      const float w = decay(rl, cnt);
      sum *= w;
#pragma unroll
      for (int ct = 0; ct < DT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) S[ct][e] *= w;
    }
    for (int b0 = 0; 32 * b0 < cnt; b0 += PB) {
      __syncthreads();
      for (int blk = wave; blk < PB; blk += waves) {
        const int r = 32 * (b0 + blk) + lr;
        uint4 xf[DK][NSX];
        const double sq = load_x<TX, DK>(k + static_cast<size_t>(p0 + min(r, cnt - 1)) * d, r < cnt, d, xf);
#pragma unroll
        for (int ks = 0; ks < DK; ++ks)
#pragma unroll
          for (int s = 0; s < NSX; ++s) xl[((blk * DK + ks) * NSX + s) * kFragLanes + lane] = xf[ks][s];
        if (lh == 0) {
          // the weight of the chunk's end, e^{-rate (cnt - 1 - r)}, goes with the row's factors
          RowFactors o = row_factors<ELU>(sq, a.nprf, a.log2_m);
          const float e = -rl * static_cast<float>(REV ? r : cnt - 1 - r);
          if (ELU)
            o.f = r < cnt ? __builtin_amdgcn_exp2f(e) : 0.f;
          else
            o.c = r < cnt ? o.c + e : -INFINITY;
          fr[32 * blk + lr] = o.r, fc[32 * blk + lr] = o.c, ff[32 * blk + lr] = o.f;
          if (REV) fd[32 * blk + lr] = r < cnt ? a.gd[static_cast<size_t>(bh) * a.n + p0 + r] : 0.f;
        }
      }
      stage_columns<TV, DT, NV, Values::kAsIs>(v, p0 + 32 * b0, cnt - 32 * b0, d, PB, vl, nullptr);
      __syncthreads();
      for (int blk = 0; blk < PB && 32 * (b0 + blk) < cnt; ++blk) {
        floatx16 acc = zero16(), lo = zero16();
#pragma unroll
        for (int ks = 0; ks < DK; ++ks) {
          uint4 x[NSX];
          read_terms<NSX>(xl + (blk * DK + ks) * NSX * kFragLanes, x);
#pragma unroll
          for (int s = 2; s >= 1; --s)
#pragma unroll
            for (int i = 0; i <= s; ++i)
              if (s - i < NSX) lo = mfma_bf16(x[s - i], wf[ks][i], lo);
          acc = mfma_bf16(x[0], wf[ks][0], acc);
        }
        floatx16 ph;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int at = 32 * blk + 8 * g + 4 * lh;
          const float4 r4 = *reinterpret_cast<const float4*>(fr + at), c4 = *reinterpret_cast<const float4*>(fc + at),
                       f4 = *reinterpret_cast<const float4*>(ff + at);
          ph[4 * g] = feature<ELU>(acc[4 * g], lo[4 * g], r4.x, c4.x, f4.x);
          ph[4 * g + 1] = feature<ELU>(acc[4 * g + 1], lo[4 * g + 1], r4.y, c4.y, f4.y);
          ph[4 * g + 2] = feature<ELU>(acc[4 * g + 2], lo[4 * g + 2], r4.z, c4.z, f4.z);
          ph[4 * g + 3] = feature<ELU>(acc[4 * g + 3], lo[4 * g + 3], r4.w, c4.w, f4.w);
        }
        if (l >= a.M) ph = zero16();
#pragma unroll
        for (int e = 0; e < 16; ++e)
          sum = REV ? fmaf(ph[e], fd[32 * blk + 8 * (e >> 2) + 4 * lh + (e & 3)], sum) : sum + ph[e];
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          uint4 pf[NP];
          pack_half<NP>(ph, k2, pf);
#pragma unroll
          for (int ct = 0; ct < DT; ++ct) {
            uint4 vf[NV];
            read_terms<NV>(vl + ((blk * DT + ct) * 2 + k2) * NV * kFragLanes, vf);
            S[ct] = mfma_terms<NV, NP>(vf, pf, S[ct]);
          }
        }
      }
    }
  }
  store((REV ? a.totb : a.tot) + (static_cast<size_t>(bh) * a.nseg + seg) * cells);
}

// (REV: after each segment.)  The state before each segment, in place of the segment's sums, and the one
// behind the sequence: A <- e^{-rate rows} A + sums, one thread an element.
template <bool REV>
__global__ __launch_bounds__(256) void k_decay_join(DecayArgs a) {
  const int bh = blockIdx.x, b = bh / a.H, h = bh % a.H;
  const int cells = (a.d + 1) * a.Mp;
  const int slot = !REV && a.state ? slot_of(a.slots, b, a.B, a.nslots) : kStateNone;
  const int e = blockIdx.y * 256 + threadIdx.x;
  if (e >= cells) return;
  const int c = e / a.Mp, l = e % a.Mp;
  const float rl = rate_log2(a.rate[h]);
  const int rows = rows_of(a.lens, b, a.n);
  float* st = slot >= 0 && l < a.M ? a.state + ((static_cast<size_t>(slot) * a.H + h) * (a.d + 1) + c) * a.M + l : nullptr;
  float s = st && !a.fresh ? *st : 0.f;
  float* __restrict__ t = (REV ? a.totb : a.tot) + static_cast<size_t>(bh) * a.nseg * cells + e;
  const int per = a.segc * kChunk;
  for (int s0 = 0; s0 < a.nseg; ++s0) {
    const int g = REV ? a.nseg - 1 - s0 : s0;
    const float sums = t[static_cast<size_t>(g) * cells];
    t[static_cast<size_t>(g) * cells] = s;
    const int cnt = min(max(rows - g * per, 0), per);
    s = cnt ? fmaf(decay(rl, cnt), s, sums) : s;
  }
  if (st) *st = s;
}


// NP, NV: terms of the features and of the values.
template <typename TX, typename TV, int DK, int NP, int NV, bool ELU, bool REV>
void launch_decay_states(const DecayArgs& a, hipStream_t st) {
  constexpr int NSX = kTermsX<TX>, DT = DK / 2, PB = NSX == 3 && DK == 8 ? 2 : 4;
  constexpr int lds = PB * (DK * NSX + DT * 2 * NV) * 1024;
  if constexpr (lds > 65536)
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&k_decay_states<TX, TV, DK, NP, NV, ELU, REV>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  const int BH = a.B * a.H, waves = a.Mp / 32 < 4 ? a.Mp / 32 : 4;
  const dim3 grid(BH, a.nseg, (a.Mp / 32 + waves - 1) / waves);
  hipLaunchKernelGGL((k_decay_states<TX, TV, DK, NP, NV, ELU, REV>), grid, dim3(64 * waves), lds, st, a);
  hipLaunchKernelGGL(k_decay_join<REV>, dim3(BH, ((a.d + 1) * a.Mp + 255) / 256), dim3(256), 0, st, a);
}

}  // namespace krpe
