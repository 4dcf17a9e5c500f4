// Attention with a bias that decays, b_t = rate t for t <= 0 and -inf after:
// Eq. (10) over a state,
//
//   num_i | den_i = sum_{j <= i} e^{-rate (i - j)} (phi(q_i) . phi(k_j)) [v_j | 1]
//                 = A_i phi(q_i),   A_i = e^{-rate} A_{i-1} + [v_i; 1] phi(k_i)^T
//
// A is [d + 1, M]: numerators of the d value columns, then the denominators.
// Shared by the prompts' kernels (decay_fwd.hip), their gradients
// (decay_bwd.hip), the single tokens (decay_step.hip) and the drafted trees
// (decay_tree.hip).
//
// Operands are bf16 terms in the fragments of wprod.hpp, which have fp32's range
// and need no scale: three terms hold an fp32 value whole, two to 2.6e-6 of it
// (rms), one to 1.7e-3.  Where the result is fp32 (states always, z and the
// gradients with fp32 inputs) every operand has three terms and a product of
// two takes the six of at least 2^-16 of it.  Where the result is rounded to
// bf16 (1.7e-3 by itself), features have one term, whose errors average over
// them, and the weights P and the state, whose errors would add to it, two.
// Projections take W in three terms (two for bf16 results): an error of the
// exponent is one of phi.  All sums are fp32.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "features.hpp"
#include "wprod.hpp"

namespace krpe {

constexpr int kChunk = 128;  // positions of a chunk: four row tiles of 32
constexpr int kStateNone = -1, kStateBad = -2;

// The pool's row of sequence b: kStateNone for a negative slot of -1 (no state:
// zeros before, not kept), kStateBad for one outside the pool or named by another
// sequence of the call too (two would write one state).  Every lane gets it.
__device__ __forceinline__ int slot_of(const int* __restrict__ slots, int b, int B, int nslots) {
  if (!slots) return b;
  const int s = slots[b];
  if (s == -1) return kStateNone;
  if (s < 0 || s >= nslots) return kStateBad;
  int twice = 0;
  for (int j = threadIdx.x & 63; j < B; j += 64) twice |= j != b && slots[j] == s;
  return __any(twice) ? kStateBad : s;
}

// (a rate of inf weighs 1 at distance 0 and 0 beyond)
__device__ __forceinline__ float rate_log2(float rate) { return (rate > 1e6f ? 1e6f : rate) * 1.44269504f; }
__device__ __forceinline__ float decay(float rl, int dist) { return __builtin_amdgcn_exp2f(-rl * static_cast<float>(dist)); }

// ---- rows of x as operands
template <typename TX>
constexpr int kTermsX = sizeof(TX) == 2 ? 1 : 3;

// A lane's row (dimensions 16 ks + 8 lh + t) and its squared norm in fp64; zeros where !ok.
template <typename TX, int DK>
__device__ __forceinline__ double load_x(const TX* __restrict__ row, bool ok, int d, uint4 (&xf)[DK][kTermsX<TX>]) {
  const int lh = (threadIdx.x & 63) >> 5;
  const bool vec = d % 8 == 0;
  double sq = 0.0;
#pragma unroll
  for (int ks = 0; ks < DK; ++ks) {
    const int c = 16 * ks + 8 * lh;
    float v8[8];
    load8(row + (c < d ? c : 0), ok ? d - c : 0, vec, v8);
#pragma unroll
    for (int t = 0; t < 8; ++t) sq = fma(static_cast<double>(v8[t]), static_cast<double>(v8[t]), sq);
    if constexpr (kTermsX<TX> == 1) {
      xf[ks][0] = make_uint4(pack_bf16(floatx2{v8[0], v8[1]}), pack_bf16(floatx2{v8[2], v8[3]}), pack_bf16(floatx2{v8[4], v8[5]}),
                             pack_bf16(floatx2{v8[6], v8[7]}));
    } else {
      split_bf16x8(v8, xf[ks]);
    }
  }
  return sq + __shfl_xor(sq, 32);
}

// What phi takes of a row: PRF phi_prf's r, c, f (features.hpp); elu + 1: the row's scale and 1.
struct RowFactors {
  float r, c, f;
};
template <bool ELU>
__device__ __forceinline__ RowFactors row_factors(double sq, bool nprf, double log2_m) {
  const bool nz = sq > 0.0;
  const double scale = nprf ? (nz ? 1.0 / sqrt(sq) : 0.0) : 1.0;
  RowFactors o;
  if constexpr (ELU) {
    o.r = static_cast<float>(scale), o.c = 0.f, o.f = 1.f;
  } else {
    const double c = log2_m - (nprf ? (nz ? 0.5 : 0.0) : 0.5 * sq) * kLog2e;
    o.r = static_cast<float>(scale * kLog2e), o.c = static_cast<float>(c);
    o.f = rounding_factor(c, o.c);
  }
  return o;
}
template <bool ELU>
__device__ __forceinline__ float feature(float s, float sl, float r, float c, float f) {
  if constexpr (ELU) {
    const float x = (s + sl) * r;
    return (x > 0.f ? x + 1.f : __builtin_amdgcn_exp2f(x * 1.44269504f)) * f;
  } else {
    return phi_prf(s, sl, r, c, f);
  }
}

// 32 rows of W from f0 as operands wf[ks][term][64] in LDS (zeros past m; elu + 1: rows of the identity).
template <int DK, int NW, bool ELU>
__device__ __forceinline__ void stage_weights(const float* __restrict__ W, int f0, int m, int d, uint4* __restrict__ wf) {
  for (int e = threadIdx.x; e < 32 * 2 * DK; e += blockDim.x) {
    const int fl = e / (2 * DK), c = e % (2 * DK), f = f0 + fl;
    float v8[8];
    if constexpr (ELU) {
#pragma unroll
      for (int t = 0; t < 8; ++t) v8[t] = 8 * c + t == f ? 1.f : 0.f;
    } else {
      load8(W + static_cast<size_t>(min(f, m - 1)) * d + min(8 * c, d - 1), f < m ? d - 8 * c : 0, d % 4 == 0, v8);
    }
    uint4 t3[3];
    split_bf16x8(v8, t3);
    uint4* __restrict__ o = wf + (c >> 1) * NW * kFragLanes + (c & 1) * 32 + fl;
#pragma unroll
    for (int s = 0; s < NW; ++s) o[s * kFragLanes] = t3[s];
  }
}

// Projections of 32 rows on 32 features (project of features.hpp with NW terms of W): the
// products of the largest terms and the others apart.
template <int DK, int NSX, int NW, bool XROWS>
__device__ __forceinline__ void project_terms(const uint4* __restrict__ wf, const uint4 (&xf)[DK][NSX], floatx16& acc,
                                              floatx16& lo) {
  const int lane = threadIdx.x & 63;
  acc = zero16();
  lo = zero16();
  auto mul = [](uint4 w, uint4 x, floatx16 c) { return XROWS ? mfma_bf16(x, w, c) : mfma_bf16(w, x, c); };
#pragma unroll
  for (int ks = 0; ks < DK; ++ks) {
    uint4 w[NW];
#pragma unroll
    for (int s = 0; s < NW; ++s) w[s] = wf[(ks * NW + s) * kFragLanes + lane];
#pragma unroll
    for (int s = 2; s >= 1; --s)
#pragma unroll
      for (int i = 0; i <= s; ++i)
        if (i < NW && s - i < NSX) lo = mul(w[i], xf[ks][s - i], lo);
    acc = mul(w[0], xf[ks][0], acc);
  }
}

// ---- NT terms of computed operands, and their products
template <int NT>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&t)[NT]) {
  floatx2 v;
  v.x = a;
  v.y = b;
  t[0] = pack_bf16(v);
  if constexpr (NT >= 2) {
    v = minus_bf16(v, t[0]);
    t[1] = pack_bf16(v);
  }
  if constexpr (NT == 3) t[2] = pack_bf16(minus_bf16(v, t[1]));
}
// Registers 8 h .. 8 h + 7 of a 32 x 32 result as the fragment of its k step h.
template <int NT>
__device__ __forceinline__ void pack_half(const floatx16& x, int h, uint4 (&t)[NT]) {
  uint32_t p[4][NT];
#pragma unroll
  for (int j = 0; j < 4; ++j) split_pair<NT>(x[8 * h + 2 * j], x[8 * h + 2 * j + 1], p[j]);
#pragma unroll
  for (int s = 0; s < NT; ++s) t[s] = make_uint4(p[0][s], p[1][s], p[2][s], p[3][s]);
}
// The products of terms s and t with s + t < max(NA, NB), the small ones first.
template <int NA, int NB>
__device__ __forceinline__ floatx16 mfma_terms(const uint4 (&a)[NA], const uint4 (&b)[NB], floatx16 c) {
  constexpr int most = NA > NB ? NA : NB;
#pragma unroll
  for (int s = most - 1; s >= 0; --s)
#pragma unroll
    for (int i = 0; i <= s; ++i)
      if (i < NA && s - i < NB) c = mfma_bf16(a[i], b[s - i], c);
  return c;
}
template <int N>
__device__ __forceinline__ void read_terms(const uint4* __restrict__ p, uint4 (&t)[N]) {
#pragma unroll
  for (int s = 0; s < N; ++s) t[s] = p[s * kFragLanes + (threadIdx.x & 63)];
}

// Four values of a row from column c (zeros past d, or all of them where !ok).
template <typename TX>
__device__ __forceinline__ void load4(const TX* __restrict__ row, int c, bool ok, int d, float (&v)[4]) {
  if (ok && d % 4 == 0 && c < d) {
    if constexpr (std::is_same<TX, float>::value) {
      const float4 u = *reinterpret_cast<const float4*>(row + c);
      v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(row + c);
      v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xffff0000u);
      v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = ok && c + t < d ? to_f32(row[c + t]) : 0.f;
  }
}
template <typename TZ>
__device__ __forceinline__ void store4(TZ* __restrict__ row, int c, int d, const float (&v)[4]) {
  if (d % 4 == 0 && c < d) {
    if constexpr (std::is_same<TZ, float>::value)
      *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
    else
      *reinterpret_cast<uint2*>(row + c) = make_uint2(pack_bf16(floatx2{v[0], v[1]}), pack_bf16(floatx2{v[2], v[3]}));
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (c + t < d) {
        if constexpr (std::is_same<TZ, float>::value)
          row[c + t] = v[t];
        else
          row[c + t] = static_cast<uint16_t>(pack_bf16(floatx2{v[t], 0.f}));
      }
  }
}

__device__ __forceinline__ bool finite(float v) { return fabsf(v) <= 3.4028235e38f; }

// Rows p0 .. p0 + 32 blocks - 1 of a [.][d] array turned into Z fragments (column 32 ct + lr,
// positions along the slots) vf[block][ct][k2][term][64], zeros past `rows` rows and past d.
// CLEAN: a value that is not finite goes in as zero and sets *odd, as a product with a weight of
// zero would carry it to rows that do not see it; MARK: 1 for such values and 0 for others.
enum class Values { kAsIs, kClean, kMark };
template <typename TX, int DT, int NT, Values MODE>
__device__ __forceinline__ void stage_columns(const TX* __restrict__ v, int p0, int rows, int d, int blocks,
                                              uint4* __restrict__ vf, int* __restrict__ odd) {
  for (int e = threadIdx.x; e < blocks * 8 * DT * 8; e += blockDim.x) {
    const int cg = e % (DT * 8), g = (e / (DT * 8)) % 8, blk = e / (DT * 64);
    const int c = 4 * cg, r0 = 32 * blk + 4 * g;
    float val[4][4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
      load4(v + static_cast<size_t>(p0 + min(r0 + r, rows - 1)) * d, c, r0 + r < rows, d, val[r]);
    if constexpr (MODE != Values::kAsIs) {
      bool bad = false;
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const bool f = finite(val[r][t]);
          bad |= !f;
          if constexpr (MODE == Values::kMark)
            val[r][t] = f ? 0.f : 1.f;
          else
            val[r][t] = f ? val[r][t] : 0.f;
        }
      if (MODE == Values::kClean && bad) *odd = 1;
    }
    uint2* __restrict__ o = reinterpret_cast<uint2*>(
        vf + (((blk * DT + (c >> 5)) * 2 + (g >> 2)) * NT) * kFragLanes + (g & 1) * 32 + (c & 31));
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      uint32_t a[NT], b[NT];
      split_pair<NT>(val[0][t], val[1][t], a);
      split_pair<NT>(val[2][t], val[3][t], b);
#pragma unroll
      for (int s = 0; s < NT; ++s) o[2 * (s * kFragLanes + t) + ((g >> 1) & 1)] = make_uint2(a[s], b[s]);
    }
  }
}

// ---- the prompts' passes
struct DecayArgs {
  const void *q, *k, *v;
  void* z;
  const float *rate, *W;
  float* state;         // pool [nslots][H][d + 1][M], or NULL
  const int *slots, *lens;
  float* tot;           // [BH][nseg][d + 1][Mp]: a segment's sums at its end, then the state before it
  float* pre;           // [BH][nchunk][d + 1][Mp]: sums of the segment before each of its chunks
  // gradients: dz; dq, dk, dv; [dL/dnumerators | dL/ddenominator] of the rows, g [BH][n][d] and
  // gd [BH][n]; the queries' sums backwards in time, totb and preb as tot and pre
  const void* dz;
  void *dq, *dk, *dv;
  float *g, *gd, *totb, *preb;
  int B, H, n, d, M, Mp, nchunk, nseg, segc, nslots, nprf, fresh;
  double log2_m;
};
// ---- calls on a pool of states
struct PoolArgs {
  const void *q, *k, *v;
  void* z;
  const float *rate, *W;
  float* state;             // [nslots][H][d + 1][M]
  const int *slots, *tree;  // tree: parents [B][T] (tree), accepted nodes [B][P] (commit)
  int B, H, T, P, d, M, nslots, nprf;
  float log_m;              // -log(sqrt(m))
  double log2_m;            // -log2(sqrt(m))
};
__device__ __forceinline__ int rows_of(const int* __restrict__ lens, int b, int n) {
  return lens ? min(max(lens[b], 0), n) : n;
}

// Host-side launchers (decay_fwd.hip, decay_bwd.hip, decay_step.hip, decay_tree.hip).
hipError_t launch_decay_fwd(bool bf16, bool elu, const DecayArgs& a, hipStream_t st);
hipError_t launch_decay_bwd(bool bf16, bool elu, const DecayArgs& a, hipStream_t st);
hipError_t launch_decay_step(bool bf16, bool elu, const PoolArgs& a, hipStream_t st);
hipError_t launch_decay_tree(bool bf16, bool elu, const PoolArgs& a, hipStream_t st);
hipError_t launch_decay_commit(bool bf16, bool elu, const PoolArgs& a, hipStream_t st);
hipError_t launch_state_copy(float* state, const int* src, const int* dst, int count, int nslots, long long cells,
                             hipStream_t st);

}  // namespace krpe
