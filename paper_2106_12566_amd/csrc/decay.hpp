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
// Projections take W in three terms (two for bf16 results) and bf16 rows as
// they are: an error of the exponent is one of phi.  fp32 rows, brought below 1
// by a power of two, and W are two fp16 terms, 2^-23 of an element each, and
// three products (|W| < 65504).  All sums are fp32.
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

// The pool's row of sequence b: kStateNone for a negative slot of -1 (no state: zeros before, not
// kept), kStateBad for one outside the pool or named by another sequence of the call too (two
// would write one state).  Every lane gets it.  slot_in() leaves the last to check_slot(), so that
// a state can be asked for, not written, before the other sequences' slots are there.
__device__ __forceinline__ int slot_in(const int* __restrict__ slots, int b, int nslots) {
  if (!slots) return b;
  const int s = slots[b];
  return s == -1 ? kStateNone : (s < 0 || s >= nslots ? kStateBad : s);
}
__device__ __forceinline__ int check_slot(const int* __restrict__ slots, int slot, int b, int B) {
  if (!slots || slot < 0) return slot;
  int twice = 0;
  for (int j = threadIdx.x & 63; j < B; j += 64) twice |= j != b && slots[j] == slot;
  return __any(twice) ? kStateBad : slot;
}
__device__ __forceinline__ int slot_of(const int* __restrict__ slots, int b, int B, int nslots) {
  return check_slot(slots, slot_in(slots, b, nslots), b, B);
}

// (a rate of inf weighs 1 at distance 0 and 0 beyond)
__device__ __forceinline__ float rate_log2(float rate) { return (rate > 1e6f ? 1e6f : rate) * 1.44269504f; }
__device__ __forceinline__ float decay(float rl, int dist) { return __builtin_amdgcn_exp2f(-rl * static_cast<float>(dist)); }

// The weights e^{-rate dist} of a 32 x 32 result's rows: dist = sign (i - j) for the lane's row i and rows
// j = base + 8 (e / 4) + 4 lh + e % 4 along the registers; zero below 0 (EDGE: where that can be).
// There each by itself; elsewhere as products of the weight of the nearest of each four rows and one of
// four that all share, which are in range wherever the weight is.
struct TileWeights {
  float rl;
  int sign;
  float t[4];
  __device__ __forceinline__ TileWeights(float rl_, int sign_) : rl(rl_), sign(sign_) {
#pragma unroll
    for (int j = 0; j < 4; ++j) t[j] = decay(rl, sign > 0 ? 3 - j : j);
  }
  template <bool EDGE>
  __device__ __forceinline__ void apply(floatx16& x, int i, int base) const {
    const int d0 = sign * (i - base - 4 * static_cast<int>((threadIdx.x & 63) >> 5));
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float w = EDGE ? 0.f : decay(rl, d0 - sign * 8 * g - (sign > 0 ? 3 : 0));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (EDGE) {
          const int dist = d0 - sign * (8 * g + j);
          const float y = x[4 * g + j] * decay(rl, dist);
          x[4 * g + j] = dist > 0 ? y : (dist == 0 ? x[4 * g + j] : 0.f);
        } else {
          x[4 * g + j] *= w * t[j];
        }
      }
    }
  }
};

// ---- rows of x as operands
template <typename TX>
constexpr int kTermsX = sizeof(TX) == 2 ? 1 : 2;

// Reads of rows of d elements through a buffer resource: offsets are in bytes from `base`, and what
// lies at `bytes` or beyond (kOut among it) reads as zero.
constexpr uint32_t kOut = 0x80000000u;
template <typename T>
struct Rows {
  __amdgpu_buffer_rsrc_t r;
  int d;
  __device__ __forceinline__ Rows(const T* base, size_t count, int d_) : r(buffer_of(base, count * d_ * sizeof(T))), d(d_) {}
  __device__ __forceinline__ uint32_t at(int row) const { return static_cast<uint32_t>(row) * static_cast<uint32_t>(d) * sizeof(T); }
  // element c of the row at o (kOut past the row)
  __device__ __forceinline__ uint32_t at(uint32_t o, int c) const { return c < d ? o + c * sizeof(T) : kOut; }
  __device__ __forceinline__ float one(uint32_t o) const {
    if constexpr (sizeof(T) == 2)
      return to_f32(static_cast<uint16_t>(__builtin_amdgcn_raw_buffer_load_b16(r, o, 0, 0)));
    else
      return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, o, 0, 0));
  }
  __device__ __forceinline__ uint4 b128(uint32_t o) const {
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0));
  }
  __device__ __forceinline__ uint2 b64(uint32_t o) const {
    return __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(r, o, 0, 0));
  }
};

// Four elements from c of the row at o as they lie in memory (zeros past d).
template <typename TX>
struct Raw4 {
  typename std::conditional<sizeof(TX) == 2, uint2, uint4>::type u;
  __device__ __forceinline__ void load(const Rows<TX>& x, uint32_t o, int c) {
    o = x.at(o, c);
    if (x.d % 4 == 0) {
      if constexpr (sizeof(TX) == 2)
        u = x.b64(o);
      else
        u = x.b128(o);
    } else {
      float v[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        v[t] = x.one(o + t * sizeof(TX));
        v[t] = c + t < x.d ? v[t] : 0.f;
      }
      if constexpr (sizeof(TX) == 2)
        u = make_uint2(pack_bf16(floatx2{v[0], v[1]}), pack_bf16(floatx2{v[2], v[3]}));
      else
        u = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
  }
  __device__ __forceinline__ void values(float (&v)[4]) const {
    if constexpr (sizeof(TX) == 2) {
      v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xffff0000u);
      v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xffff0000u);
    } else {
      v[0] = __uint_as_float(u.x), v[1] = __uint_as_float(u.y), v[2] = __uint_as_float(u.z), v[3] = __uint_as_float(u.w);
    }
  }
};
template <typename TX>
__device__ __forceinline__ void load4(const Rows<TX>& x, uint32_t o, int c, float (&v)[4]) {
  Raw4<TX> r;
  r.load(x, o, c);
  r.values(v);
}
// Eight elements from c of the row at o as they lie in memory (zeros past d).
template <typename TX>
struct Raw8 {
  uint4 u[sizeof(TX) / 2];
  __device__ __forceinline__ void load(const Rows<TX>& x, uint32_t o, int c) {
    o = x.at(o, c);
    if (x.d % 8 == 0) {
#pragma unroll
      for (int i = 0; i < static_cast<int>(sizeof(TX) / 2); ++i) u[i] = x.b128(o + 16 * i);
    } else {
      float v[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        v[t] = x.one(o + t * sizeof(TX));
        v[t] = c + t < x.d ? v[t] : 0.f;
      }
      if constexpr (sizeof(TX) == 2) {
        u[0] = make_uint4(pack_bf16(floatx2{v[0], v[1]}), pack_bf16(floatx2{v[2], v[3]}), pack_bf16(floatx2{v[4], v[5]}),
                          pack_bf16(floatx2{v[6], v[7]}));
      } else {
        u[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        u[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
      }
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    if constexpr (sizeof(TX) == 2) {
      const unsigned w[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) v[2 * j] = __uint_as_float(w[j] << 16), v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    } else {
      const unsigned w[8] = {u[0].x, u[0].y, u[0].z, u[0].w, u[1].x, u[1].y, u[1].z, u[1].w};
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
    }
  }
  // the operand's terms (bf16: the elements themselves; fp32: those of scale times them)
  __device__ __forceinline__ void terms(float scale, uint4 (&t)[kTermsX<TX>]) const {
    if constexpr (sizeof(TX) == 2) {
      t[0] = u[0];
    } else {
      float v[8];
      values(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= scale;
      split_f16x8(v, kLoScale, t[0], t[1]);
    }
  }
};
// A lane's row at o (dimensions 16 ks + 8 lh + t), fetched.
template <typename TX, int DK>
__device__ __forceinline__ void fetch_row(const Rows<TX>& rows, uint32_t o, Raw8<TX> (&x)[DK]) {
  const int lh = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int ks = 0; ks < DK; ++ks) x[ks].load(rows, o, 16 * ks + 8 * lh);
}
// Its squared norm (it is the same for every feature: an error of it weighs on the whole position), in
// sixteen partial sums added in fp64.
template <typename TX, int DK>
__device__ __forceinline__ double row_square(const Raw8<TX> (&x)[DK]) {
  float p[8] = {};
#pragma unroll
  for (int ks = 0; ks < DK; ++ks) {
    float v[8];
    x[ks].values(v);
#pragma unroll
    for (int t = 0; t < 8; ++t) p[t] = fmaf(v[t], v[t], p[t]);
  }
  double s = p[0];
#pragma unroll
  for (int t = 1; t < 8; ++t) s += static_cast<double>(p[t]);
  return s + __shfl_xor(s, 32);
}

// What phi takes of a row: PRF 2^(s r + c) of the projection s, r = log2(e) (over ||x|| when
// normalising), c = -||x||^2 / 2 log2(e) - log2(sqrt(m)); elu + 1 r alone.  f: what the rounding of c
// left, as a part of s (of its accumulator lo; for the states, it weighs little on a ratio).  x: what the operand's terms were scaled by (fp32
// rows: a power of two that brings them below 1, which r makes good).
struct RowFactors {
  float r, c, f, x;
};
template <bool ELU, bool WHOLE>
__device__ __forceinline__ RowFactors row_factors(double sq, bool nprf, double log2_m) {
  const bool nz = sq > 0.0;
  const float norm = sqrtf(static_cast<float>(sq));
  RowFactors o;
  o.r = (ELU ? 1.f : static_cast<float>(kLog2e)) * (nprf ? (nz ? 1.f / norm : 0.f) : 1.f);
  const double c = log2_m - (nprf ? (nz ? 0.5 : 0.0) : 0.5 * sq) * kLog2e;
  o.c = static_cast<float>(c);
  o.f = 0.f;
  o.x = 1.f;
  if constexpr (WHOLE) {
    const unsigned n = __float_as_uint(norm) >> 23;  // |x| < 2^(n - 126)
    const unsigned e = nz ? min(max(n, 2u), 252u) : 126u;
    o.x = __uint_as_float((253u - e) << 23);
    o.r *= __uint_as_float((e + 1u) << 23);
  }
  if (!ELU && nz && isfinite(o.c)) o.f = static_cast<float>(c - static_cast<double>(o.c)) / o.r * (WHOLE ? kLoScale : 1.f);
  return o;
}
// WHOLE: the projection in two accumulators, lo in units of 2^-11 (fp32 rows).
template <bool ELU, bool WHOLE>
__device__ __forceinline__ float feature(float s, float sl, float r, float c) {
  if constexpr (WHOLE) s = fmaf(sl, kLoInv, s);
  if constexpr (ELU) {
    const float x = s * r;
    return x > 0.f ? x + 1.f : __builtin_amdgcn_exp2f(x * 1.44269504f);
  } else {
    return __builtin_amdgcn_exp2f(fmaf(s, r, c));
  }
}

// 32 rows of W from f0 as operands wf[ks][term][64] in LDS (zeros past m; elu + 1: rows of the
// identity), fetched by a work-group of 256 threads and put a step later.
// (W's rows past m read as zeros)
template <bool ELU>
__device__ __forceinline__ void load_weights(const Rows<float>& W, int f, int c, float (&v)[8]) {
  if constexpr (ELU) {
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = c + t == f ? 1.f : 0.f;
  } else {
    float u[4];
    load4(W, W.at(f), c, u);
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = u[t];
    load4(W, W.at(f), c + 4, u);
#pragma unroll
    for (int t = 0; t < 4; ++t) v[4 + t] = u[t];
  }
}
// Eight of its elements as operand terms: NW bf16 ones, or (WHOLE) two fp16 ones.
template <int NW, bool WHOLE>
__device__ __forceinline__ void weight_terms(const float (&v)[8], uint4 (&t)[NW]) {
  if constexpr (WHOLE) {
    static_assert(NW == 2, "two fp16 terms");
    split_f16x8(v, kLoScale, t[0], t[1]);
  } else {
    uint4 t3[3];
    split_bf16x8(v, t3);
#pragma unroll
    for (int s = 0; s < NW; ++s) t[s] = t3[s];
  }
}
template <int DK, int NW, bool ELU, bool WHOLE>
struct WeightTile {
  static constexpr int N = (64 * DK + 255) / 256;
  float v[N][8];
  __device__ __forceinline__ void fetch(const Rows<float>& W, int f0) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = threadIdx.x + 256 * i;
      if (N * 256 > 64 * DK && e >= 64 * DK) return;
      load_weights<ELU>(W, f0 + (e & 31), 8 * (e >> 5), v[i]);
    }
  }
  __device__ __forceinline__ void put(uint4* __restrict__ wf) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = threadIdx.x + 256 * i, fl = e & 31, c = e >> 5;
      if (N * 256 > 64 * DK && e >= 64 * DK) return;
      uint4 t[NW];
      weight_terms<NW, WHOLE>(v[i], t);
      uint4* __restrict__ o = wf + (c >> 1) * NW * kFragLanes + (c & 1) * 32 + fl;
#pragma unroll
      for (int s = 0; s < NW; ++s) o[s * kFragLanes] = t[s];
    }
  }
};

// Projections of 32 rows on 32 features: with WHOLE h h (acc) and h l + l h (lo, in units of 2^-11)
// apart; products of bf16 terms in one sum, the small ones first, or with three terms of W the first
// one's (acc) apart from the others (lo), so that the large sum takes few roundings.  lo comes with
// what it begins with (the rows' f).
template <int DK, int NSX, int NW, bool XROWS, bool WHOLE, typename FW, typename FX>
__device__ __forceinline__ void project_terms(FW&& weights, FX&& rows, floatx16& acc, floatx16& lo) {
  acc = zero16();
  auto mul = [](uint4 w, uint4 x, floatx16 c) {
    if constexpr (WHOLE)
      return XROWS ? mfma_f16(x, w, c) : mfma_f16(w, x, c);
    else
      return XROWS ? mfma_bf16(x, w, c) : mfma_bf16(w, x, c);
  };
#pragma unroll
  for (int ks = 0; ks < DK; ++ks) {
    uint4 w[NW], x[NSX];
    weights(ks, w);
    rows(ks, x);
    if constexpr (WHOLE) {
      lo = mul(w[0], x[1], lo);
      lo = mul(w[1], x[0], lo);
    } else {
#pragma unroll
      for (int s = NW - 1; s >= 1; --s) {
        if constexpr (NW == 3)
          lo = mul(w[s], x[0], lo);
        else
          acc = mul(w[s], x[0], acc);
      }
    }
    acc = mul(w[0], x[0], acc);
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

// Rows of a [.][d] array turned into Z fragments (column 32 ct + lr, positions along the slots)
// vf[block][ct][k2][term][64], zeros past the array's end and past d: patches of four rows and four
// columns, fetched by a work-group of THREADS and put a step later.
// kClean: a value that is not finite goes in as zero and sets *odd, as a product with a weight of
// zero would carry it to rows that do not see it; kMark: 1 for such values and 0 for others.
enum class Values { kAsIs, kClean, kMark };
template <typename TX, int DT, int BLOCKS, int THREADS>
struct ColumnTile {
  static constexpr int N = (BLOCKS * 64 * DT + THREADS - 1) / THREADS;
  Raw4<TX> v[N][4];
  // row(r): where row r of the tile lies (kOut: zeros)
  template <typename F>
  __device__ __forceinline__ void fetch(const Rows<TX>& x, F&& row) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = threadIdx.x + THREADS * i, cg = e % (DT * 8), r0 = 4 * (e / (DT * 8));
#pragma unroll
      for (int r = 0; r < 4; ++r) v[i][r].load(x, row(r0 + r), 4 * cg);
    }
  }
  template <int NT, Values MODE>
  __device__ __forceinline__ void put(uint4* __restrict__ vf, int* __restrict__ odd) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = threadIdx.x + THREADS * i;
      const int cg = e % (DT * 8), g = (e / (DT * 8)) % 8, blk = e / (DT * 64);
      const int c = 4 * cg;
      if (N * THREADS > BLOCKS * 64 * DT && blk >= BLOCKS) return;
      float val[4][4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[i][r].values(val[r]);
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
};
template <typename TX, int DT, int BLOCKS, int NT, Values MODE>
__device__ __forceinline__ void stage_columns(const Rows<TX>& x, uint4* __restrict__ vf, int* __restrict__ odd) {
  ColumnTile<TX, DT, BLOCKS, 256> t;
  t.fetch(x, [&](int r) { return x.at(r); });
  t.template put<NT, MODE>(vf, odd);
}

// Rows [r0, r1) of an array [.][d] cleared by a work-group of 256 threads.
template <typename TZ>
__device__ __forceinline__ void clear_rows(TZ* __restrict__ z, int r0, int r1, int d) {
  for (int e = r0 * d + static_cast<int>(threadIdx.x); e < r1 * d; e += 256) z[e] = TZ{};
}

// ---- the prompts' passes
struct DecayArgs {
  const void *q, *k, *v;
  void* z;
  const float *rate, *W;
  float* state;         // pool [nslots][H][d + 1][M], or NULL
  const int *slots, *lens;
  // One segment (nseg == 1): pre [BH][nchunk][d + 1][Mp] is the state before each chunk.  More:
  // pre is the sums of the segment before each of its chunks but the first, tot [BH][nseg][d + 1][Mp]
  // a segment's sums at its end, and after the join the state before it.
  float *tot, *pre;
  const int* path;      // [B][P]: the rows of k, v to take (krpe_decay_commit)
  // gradients: dz; dq, dk, dv; [dL/dnumerator | dL/ddenominator] of the rows, g [BH][n][d] and
  // gd [BH][n]; the queries' sums backwards in time, totb and preb as tot and pre
  const void* dz;
  void *dq, *dk, *dv;
  float *g, *gd, *totb, *preb;
  int B, H, n, d, M, Mp, nchunk, nseg, segc, nslots, nprf, fresh, P, tail;  // tail: rows behind lens are cleared
  double log2_m;
};
__device__ __forceinline__ int rows_of(const int* __restrict__ lens, int b, int n) {
  return lens ? min(max(lens[b], 0), n) : n;
}

// The state outside a chunk, wold old + pre (either may be NULL), fetched 32 features at a time.
// As rows: operands sl[ct][ks][term][64], lane: column, features in the slots' order.  As columns:
// sl[ks][term][64], lane: feature, columns in the slots' order.
template <int DT, int NT, bool COLUMNS>
struct StateTile {
  static constexpr int ITEMS = DT * 128, N = (ITEMS + 255) / 256;
  const float *old, *pre;
  float wold;
  int d, Mp;
  float o[N][8], p[N][8], so, sp;
  __device__ __forceinline__ StateTile(const float* old_, const float* pre_, float w, int d_, int Mp_)
      : old(old_), pre(pre_), wold(w), d(d_), Mp(Mp_), so(0.f), sp(0.f) {}
  __device__ __forceinline__ bool any() const { return old || pre; }
  __device__ __forceinline__ void read(const float* __restrict__ from, int f0, float (&x)[N][8], float& last) const {
    const Rows<float> r(from, d + 1, Mp);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int e = threadIdx.x + 256 * n;
      if (N * 256 > ITEMS && e >= ITEMS) break;
      if constexpr (COLUMNS) {
        const int l = e & 31, half = (e >> 5) & 1, ks = e >> 6;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const int c = 16 * ks + 8 * (t >> 2) + 4 * half + (t & 3);
          x[n][t] = r.one(c < d ? r.at(c) + 4u * (f0 + l) : kOut);
        }
      } else {
        const int c = 32 * (e >> 7) + (e & 31), ks = (e >> 6) & 1, half = (e >> 5) & 1;
        const uint32_t at = c < d ? r.at(c) + 4u * (f0 + 16 * ks + 4 * half) : kOut;
        const uint4 u = r.b128(at), w = r.b128(at + 32);
        x[n][0] = __uint_as_float(u.x), x[n][1] = __uint_as_float(u.y), x[n][2] = __uint_as_float(u.z), x[n][3] = __uint_as_float(u.w);
        x[n][4] = __uint_as_float(w.x), x[n][5] = __uint_as_float(w.y), x[n][6] = __uint_as_float(w.z), x[n][7] = __uint_as_float(w.w);
      }
    }
    if (threadIdx.x < 32) last = from[static_cast<size_t>(d) * Mp + f0 + threadIdx.x];
  }
  __device__ __forceinline__ void fetch(int f0) {
    if (old) read(old, f0, o, so);
    if (pre) read(pre, f0, p, sp);
  }
  __device__ __forceinline__ void put(uint4* __restrict__ sl, float* __restrict__ sden) const {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int e = threadIdx.x + 256 * n;
      if (N * 256 > ITEMS && e >= ITEMS) break;
      float x[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) x[t] = old ? (pre ? fmaf(wold, o[n][t], p[n][t]) : wold * o[n][t]) : p[n][t];
      uint32_t q[4][NT];
#pragma unroll
      for (int j = 0; j < 4; ++j) split_pair<NT>(x[2 * j], x[2 * j + 1], q[j]);
      int at;
      if constexpr (COLUMNS)
        at = (e >> 6) * NT * kFragLanes + (e & 63);
      else
        at = (((e >> 7) * 2 + ((e >> 6) & 1)) * NT) * kFragLanes + (e & 63);
#pragma unroll
      for (int s = 0; s < NT; ++s) sl[at + s * kFragLanes] = make_uint4(q[0][s], q[1][s], q[2][s], q[3][s]);
    }
    if (threadIdx.x < 32) sden[threadIdx.x] = (old ? wold * so : 0.f) + (pre ? sp : 0.f);
  }
};

// ---- calls on a pool of states
struct PoolArgs {
  const void *q, *k, *v;
  void* z;
  const float *rate, *W;
  float* state;               // [nslots][H][d + 1][M]
  const int *slots, *parent;  // parent [B][T]
  int B, H, T, d, M, nslots, nprf;
  float log_m;                // -log(sqrt(m))
  double log2_m;              // -log2(sqrt(m))
};
// Host-side launchers (decay_fwd.hip, decay_bwd.hip, decay_step.hip, decay_tree.hip).
hipError_t launch_decay_fwd(bool bf16, bool elu, const DecayArgs& a, hipStream_t st);
hipError_t launch_decay_bwd(bool bf16, bool elu, const DecayArgs& a, hipStream_t st);
hipError_t launch_decay_step(bool bf16, bool elu, const PoolArgs& a, hipStream_t st);
hipError_t launch_decay_tree(bool bf16, bool elu, const PoolArgs& a, hipStream_t st);
hipError_t launch_decay_commit(bool bf16, bool elu, const DecayArgs& a, hipStream_t st);
hipError_t launch_state_copy(float* state, const int* src, const int* dst, int count, int nslots, long long cells,
                             hipStream_t st);

}  // namespace krpe
