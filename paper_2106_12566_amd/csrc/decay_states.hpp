// The sums of a decaying state along a sequence, forwards (the keys' [v | 1]) and
// backwards in time (the queries' gradients): by chunk within segments, then
// joined over the segments.  Used by prompts, gradients and accepted drafts.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "decay.hpp"

namespace krpe {

// kBack: the queries' sums backwards in time, of phi(q_i) [g_i | gd_i]; the rows' weights go to the
// chunk's first position, and "before" is after.  kPath: the rows path[b][0 ..] of k and v.
enum class Sums { kForth, kBack, kPath };

// The leading entries of a path that are rows (0 <= p < n); every lane gets it.
__device__ __forceinline__ int path_rows(const int* __restrict__ path, int P, int n) {
  for (int p0 = 0; p0 < P; p0 += 64) {
    const int p = p0 + (threadIdx.x & 63);
    const int at = p < P ? path[p] : -1;
    const unsigned long long none = __ballot(at < 0 || at >= n);
    if (none) return p0 + __ffsll(none) - 1;
  }
  return P;
}

// A wave owns 32 features, its sums in registers (lane: feature; value columns along the
// registers), and its W; the rows of x and v pass through LDS for all waves of the work-group,
// 32 PB of them at a time and fetched that far ahead.  (Rows in every wave's registers instead
// would be read once for each 32 features, and the sums in LDS would pass through it for each 32 rows.)
//
// Bound by waits between the matrix products: two waves a SIMD (the sums, W and the rows
// ahead take 250 registers), where the projection, exp, the split into terms and the product of a
// block follow each other.  d = 64: 96 heads, n = 4096, 128 features, fp32 (18 M d operations a row with
// the terms' products) 125 us, 0.46 PFLOP/s; 16 heads, n = 16384, 256 features, bf16 (12 M d) 88 us,
// 0.59 PFLOP/s; a large bf16 product of the library 1.22.  Three waves a SIMD spill.
// NP, NV: terms of the features and of the values.
template <typename TX, typename TV, int DK, int NP, int NV, bool ELU, Sums MODE, int WAVES>
__device__ __forceinline__ void decay_states(const DecayArgs& a, int bh, int seg, int group) {
  constexpr bool BACK = MODE == Sums::kBack, PATH = MODE == Sums::kPath, WHOLE = sizeof(TX) == 4;
  constexpr int NSX = kTermsX<TX>, NW = WHOLE ? 2 : 3, DT = DK / 2, PB = WHOLE || DK >= 6 || PATH ? 2 : 4;
  constexpr int BPW = (PB + WAVES - 1) / WAVES;  // blocks of x that a wave stages
  __shared__ __align__(16) uint4 xl[PB * DK * NSX * kFragLanes], vl[PB * DT * 2 * NV * kFragLanes];
  __shared__ __align__(16) float fr[32 * PB], fc[32 * PB], ff[32 * PB], fd[BACK ? 32 * PB : 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int b = bh / a.H, h = bh % a.H, d = a.d, M = a.M, Mp = a.Mp;
  const int l = (group * WAVES + wave) * 32 + lr;
  const int* __restrict__ path = PATH ? a.path + static_cast<size_t>(b) * a.P : nullptr;
  const int rows = PATH ? path_rows(path, a.P, a.n) : rows_of(a.lens, b, a.n);
  const bool whole = PATH || a.nseg == 1;  // uniform
  int slot = !BACK && whole && a.state ? slot_in(a.slots, b, a.nslots) : kStateNone;
  if (PATH && (slot < 0 || rows == 0)) return;
  const int c0 = PATH ? 0 : seg * a.segc, c1 = PATH ? (rows + kChunk - 1) / kChunk
                                                    : min(min(a.nchunk, c0 + a.segc), (rows + kChunk - 1) / kChunk);
  const float rl = rate_log2(a.rate[h]);
  const size_t base = static_cast<size_t>(bh) * a.n * d;
  const TX* const k = static_cast<const TX*>(BACK ? a.q : a.k) + base;
  const TV* const v = static_cast<const TV*>(BACK ? a.g : a.v) + base;
  const float* const gd = BACK ? a.gd + static_cast<size_t>(bh) * a.n : nullptr;

  Raw8<TX> rx[BPW][DK];
  ColumnTile<TV, DT, PB, 64 * WAVES> rv;
  float rd[BPW];
  // `cnt` rows from row p of the sequence (or entry p of its path), zeros after them
  auto fetch = [&](int p, int cnt) {
    const size_t from = PATH ? 0 : static_cast<size_t>(p) * d;
    const Rows<TX> xr(k + from, PATH ? a.n : cnt, d);
    const Rows<TV> vr(v + from, PATH ? a.n : cnt, d);
    auto row = [&](int r) { return PATH ? (r < cnt ? path[p + r] : -1) : r; };
#pragma unroll
    for (int i = 0; i < BPW; ++i) {
      const int r = 32 * (wave + WAVES * i) + lr;
      if (wave + WAVES * i < PB) {
        const int at = row(r);
        fetch_row<TX, DK>(xr, PATH && at < 0 ? kOut : xr.at(at), rx[i]);
        if constexpr (BACK) rd[i] = r < cnt ? gd[p + r] : 0.f;
      }
    }
    rv.fetch(vr, [&](int r) {
      const int at = row(r);
      return PATH && at < 0 ? kOut : vr.at(at);
    });
  };
  uint4 wf[DK][NW];
  {
    const Rows<float> W(a.W + static_cast<size_t>(h) * M * d, M, d);
#pragma unroll
    for (int ks = 0; ks < DK; ++ks) {
      float v8[8];
      load_weights<ELU>(W, l, 16 * ks + 8 * lh, v8);
      weight_terms<NW, WHOLE>(v8, wf[ks]);
    }
  }
  floatx16 S[DT];
  float sum = 0.f;  // the last row, of this lane half's positions
#pragma unroll
  for (int ct = 0; ct < DT; ++ct) S[ct] = zero16();
  float* __restrict__ st = slot >= 0 ? a.state + (static_cast<size_t>(slot) * a.H + h) * (d + 1) * M : nullptr;
  if (st && !a.fresh && l < M) {
#pragma unroll
    for (int ct = 0; ct < DT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int c = 32 * ct + 8 * (e >> 2) + 4 * lh + (e & 3);
        if (c < d) S[ct][e] = st[static_cast<size_t>(c) * M + l];
      }
    if (lh == 0) sum = st[static_cast<size_t>(d) * M + l];
  }
  slot = check_slot(a.slots, slot, b, a.B);
  if (PATH && slot < 0) return;
  auto store = [&](float* __restrict__ to, int width) {
    const float s = sum + __shfl_xor(sum, 32);
    if (l >= width) return;
    float* __restrict__ p = to + l + static_cast<size_t>(4 * lh) * width;
#pragma unroll
    for (int ct = 0; ct < DT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int c = 32 * ct + 8 * (e >> 2) + (e & 3);
        if (c + 4 * lh < d) p[static_cast<size_t>(c) * width] = S[ct][e];
      }
    if (lh == 0) to[static_cast<size_t>(d) * width + l] = s;
  };
  const size_t cells = static_cast<size_t>(d + 1) * Mp;
  float* const pre = BACK ? a.preb : a.pre;
  // rows q0 .. of chunk s are worked on, those of the next step fetched; s = c0 - 1: nothing yet
  auto first_of = [&](int s) { return (BACK ? c0 + c1 - 1 - s : s) * kChunk; };
#pragma unroll 1
  for (int s = c0 - 1, q0 = 0; s < c1;) {
    const int p0 = s < c0 ? 0 : first_of(s), cnt = s < c0 ? 0 : min(kChunk, rows - p0);
    if (cnt) {
      __syncthreads();  // the rows before consumed
#pragma unroll
      for (int i = 0; i < BPW; ++i) {
        const int blk = wave + WAVES * i;
        if (blk < PB) {
          RowFactors o = row_factors<ELU, WHOLE>(row_square<TX, DK>(rx[i]), a.nprf, a.log2_m);
#pragma unroll
          for (int ks = 0; ks < DK; ++ks) {
            uint4 t[NSX];
            rx[i][ks].terms(o.x, t);
#pragma unroll
            for (int n = 0; n < NSX; ++n) xl[((blk * DK + ks) * NSX + n) * kFragLanes + lane] = t[n];
          }
          if (lh == 0) {
            // the weight of the chunk's end, e^{-rate (cnt - 1 - r)}, goes with the row's factors
            const int r = q0 + 32 * blk + lr;
            // (elu + 1: as a factor in c's place)
            const float e = -rl * static_cast<float>(BACK ? r : cnt - 1 - r);
            if constexpr (ELU)
              o.c = r < cnt ? __builtin_amdgcn_exp2f(e) : 0.f;
            else
              o.c = r < cnt ? o.c + e : -INFINITY;
            fr[32 * blk + lr] = o.r, fc[32 * blk + lr] = o.c, ff[32 * blk + lr] = o.f;
            if constexpr (BACK) fd[32 * blk + lr] = rd[i];
          }
        }
      }
      rv.template put<NV, Values::kAsIs>(vl, nullptr);
    }
    const int q1 = q0 + 32 * PB < cnt ? q0 + 32 * PB : 0, s1 = q1 ? s : s + 1;
    if (s1 < c1) fetch(first_of(s1) + q1, min(32 * PB, rows - first_of(s1) - q1));
    if (cnt) {
      __syncthreads();
      if (q0 == 0) {
        if (!PATH && (s != c0 || (st && !a.fresh))) store(pre + (static_cast<size_t>(bh) * a.nchunk + p0 / kChunk) * cells, Mp);
        const float w = decay(rl, cnt);
        sum *= w;
#pragma unroll
        for (int ct = 0; ct < DT; ++ct)
#pragma unroll
          for (int e = 0; e < 16; ++e) S[ct][e] *= w;
      }
#pragma unroll 1
      for (int blk = 0; blk < PB && q0 + 32 * blk < cnt; ++blk) {
        floatx16 acc, lo, ph;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 f4 = *reinterpret_cast<const float4*>(ff + 32 * blk + 8 * g + 4 * lh);
          lo[4 * g] = f4.x, lo[4 * g + 1] = f4.y, lo[4 * g + 2] = f4.z, lo[4 * g + 3] = f4.w;
        }
        project_terms<DK, NSX, NW, true, WHOLE>(
            [&](int ks, uint4(&w)[NW]) {
#pragma unroll
              for (int n = 0; n < NW; ++n) w[n] = wf[ks][n];
            },
            [&](int ks, uint4(&x)[NSX]) { read_terms<NSX>(xl + (blk * DK + ks) * NSX * kFragLanes, x); }, acc, lo);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int at = 32 * blk + 8 * g + 4 * lh;
          const float4 r4 = *reinterpret_cast<const float4*>(fr + at), c4 = *reinterpret_cast<const float4*>(fc + at);
          const float r_[4] = {r4.x, r4.y, r4.z, r4.w}, c_[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float s = WHOLE ? acc[4 * g + j] : acc[4 * g + j] + lo[4 * g + j];
            const float y = feature<ELU, WHOLE>(s, WHOLE ? lo[4 * g + j] : 0.f, r_[j], c_[j]);
            ph[4 * g + j] = ELU ? y * c_[j] : y;
          }
        }
        if (l >= M) ph = zero16();
        if constexpr (BACK) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const float4 y = *reinterpret_cast<const float4*>(fd + 32 * blk + 8 * g + 4 * lh);
            sum = fmaf(ph[4 * g], y.x, sum), sum = fmaf(ph[4 * g + 1], y.y, sum);
            sum = fmaf(ph[4 * g + 2], y.z, sum), sum = fmaf(ph[4 * g + 3], y.w, sum);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) sum += ph[e];
        }
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
    s = s1, q0 = q1;
  }
  if (!whole)
    store((BACK ? a.totb : a.tot) + (static_cast<size_t>(bh) * a.nseg + seg) * cells, Mp);
  else if (slot >= 0)
    store(st, M);
}

template <typename TX, typename TV, int DK, int NP, int NV, bool ELU, Sums MODE, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DK <= 4 || (DK == 6 && WAVES == 4 && sizeof(TX) == 2) ? 2 : 1) void k_decay_states(DecayArgs a) {
  decay_states<TX, TV, DK, NP, NV, ELU, MODE, WAVES>(a, blockIdx.x, blockIdx.y, blockIdx.z);
}

// The state before each segment (kBack: after it) in place of the segment's sums, and the one
// behind the sequence: A <- e^{-rate rows} A + sums, one thread an element.  Bound by the latency of
// eight reads at a time: 96 heads of 65 x 128, 5 segments 11 us (32 MB), 16 of 65 x 256, 16 segments 8 us.
template <bool BACK>
__global__ __launch_bounds__(256) void k_decay_join(DecayArgs a) {
  const int bh = blockIdx.x, b = bh / a.H, h = bh % a.H;
  const int cells = (a.d + 1) * a.Mp;
  const int slot = !BACK && a.state ? slot_of(a.slots, b, a.B, a.nslots) : kStateNone;
  const int e = blockIdx.y * 256 + threadIdx.x;
  if (e >= cells) return;
  const int c = e / a.Mp, l = e % a.Mp;
  const float rl = rate_log2(a.rate[h]);
  const int rows = rows_of(a.lens, b, a.n);
  float* st = slot >= 0 && l < a.M ? a.state + ((static_cast<size_t>(slot) * a.H + h) * (a.d + 1) + c) * a.M + l : nullptr;
  float s = st && !a.fresh ? *st : 0.f;
  float* __restrict__ t = (BACK ? a.totb : a.tot) + static_cast<size_t>(bh) * a.nseg * cells + e;
  const int per = a.segc * kChunk;
  constexpr int R = 8;  // segments read at a time
  for (int s0 = 0; s0 < a.nseg; s0 += R) {
    float sums[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int g = min(s0 + r, a.nseg - 1);
      sums[r] = t[static_cast<size_t>(BACK ? a.nseg - 1 - g : g) * cells];
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (s0 + r < a.nseg) {
        const int g = BACK ? a.nseg - 1 - s0 - r : s0 + r;
        t[static_cast<size_t>(g) * cells] = s;
        const int cnt = min(max(rows - g * per, 0), per);
        s = cnt ? fmaf(decay(rl, cnt), s, sums[r]) : s;
      }
  }
  if (st) *st = s;
}

template <typename TX, typename TV, int DK, int NP, int NV, bool ELU, Sums MODE>
void launch_decay_states(const DecayArgs& a, hipStream_t st) {
  const int BH = a.B * a.H, tiles = a.Mp / 32;
  const int nseg = MODE == Sums::kPath ? 1 : a.nseg;
  if (tiles <= 2)
    hipLaunchKernelGGL((k_decay_states<TX, TV, DK, NP, NV, ELU, MODE, 2>), dim3(BH, nseg, 1), dim3(128), 0, st, a);
  else
    hipLaunchKernelGGL((k_decay_states<TX, TV, DK, NP, NV, ELU, MODE, 4>), dim3(BH, nseg, (tiles + 3) / 4), dim3(256), 0,
                       st, a);
  if (nseg > 1) {
    constexpr bool BACK = MODE == Sums::kBack;
    hipLaunchKernelGGL(k_decay_join<BACK>, dim3(BH, ((a.d + 1) * a.Mp + 255) / 256), dim3(256), 0, st, a);
  }
}

}  // namespace krpe
