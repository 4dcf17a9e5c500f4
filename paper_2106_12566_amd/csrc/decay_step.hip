// Single tokens (krpe_decay_step) and copies within a pool of states
// (krpe_decay_state_copy), both bound by the states' bytes.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "decay.hpp"

namespace krpe {

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
// Four cells of a state's row c from feature l through its buffer: what lies past the last row or the
// row's end (M) reads as zero and is not written.  NT: past the caches (the non-temporal bit).
template <bool NT>
__device__ __forceinline__ float4 load_cells(const Rows<float>& st, int c, int l, bool vec) {
  const uint32_t o = l < st.d ? st.at(c) + 4u * l : kOut;
  if (vec) {
    const uint4 u = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(st.r, o, 0, NT ? 2 : 0));
    return make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
  }
  return make_float4(st.one(o), st.one(l + 1 < st.d ? o + 4 : kOut), st.one(l + 2 < st.d ? o + 8 : kOut),
                     st.one(l + 3 < st.d ? o + 12 : kOut));
}
template <bool NT>
__device__ __forceinline__ void store_cells(const Rows<float>& st, int c, int l, bool vec, float4 v) {
  const uint32_t o = l < st.d ? st.at(c) + 4u * l : kOut;
  const uintx4 u = {__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)};
  if (vec) {
    __builtin_amdgcn_raw_buffer_store_b128(u, st.r, o, 0, NT ? 2 : 0);
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t) __builtin_amdgcn_raw_buffer_store_b32(u[t], st.r, l + t < st.d ? o + 4 * t : kOut, 0, 0);
  }
}

// One token of a sequence and head: A <- e^-rate A + [v; 1] phi(k)^T, z = A phi(q).
//
// Bound by the state, which is read and written once.  L lanes have a row's features, four each
// (256 of them at a time), and a thread K rows at a time: the first K are asked for before the
// token's features are worked out.  K sums over L lanes take fewer than K + log2(L) exchanges,
// halving at each the rows that a lane has a part of.
// 256 x 16 heads, 256 features, d = 64 (545 MB): 129 us, 4.2 TB/s, of states in memory (a plain copy 5.1).
// The same states again and again, partly from the cache: 119; with the state read after the features
// and a row summed at a time 142, with 8 or 16 rows at a time 129 and 186, with six waves a SIMD 149, as
// registers run short.
template <typename TX, int L, bool ELU, bool NT>
__global__ __launch_bounds__(256, 4) void k_decay_step(PoolArgs a) {
  constexpr int K = 4, R = 256 / L;  // rows of a thread at a time, rows side by side
  extern __shared__ __align__(16) float sm[];
  const int d = a.d, M = a.M, M4 = (M + 3) & ~3, d4 = (d + 3) & ~3;
  float *xq = sm, *xk = xq + d4, *fq = xk + d4, *fk = fq + M4, *v = fk + M4, *num = v + d4 + 4;  // v, num: d + 1
  const int b = blockIdx.x / a.H, h = blockIdx.x % a.H;
  const int lane = threadIdx.x % L, r0 = threadIdx.x / L;
  int slot = slot_in(a.slots, b, a.nslots);
  const bool vec = M % 4 == 0;
  const Rows<float> st(slot >= 0 ? a.state + (static_cast<size_t>(slot) * a.H + h) * (d + 1) * M : a.state,
                       slot >= 0 ? d + 1 : 0, M);
  const size_t row = static_cast<size_t>(blockIdx.x) * d;
  float4 u[K];
  auto fetch = [&](int l, int p) {
#pragma unroll
    for (int i = 0; i < K; ++i) u[i] = load_cells<NT>(st, (p * K + i) * R + r0, l, vec);
  };
  float sq = 0.f, sk = 0.f;  // squares of the rows, over each wave by itself
  for (int c = threadIdx.x & 63; c < d; c += 64) {
    const float y = to_f32(static_cast<const TX*>(a.q)[row + c]), x = to_f32(static_cast<const TX*>(a.k)[row + c]);
    const float w = to_f32(static_cast<const TX*>(a.v)[row + c]);
    sq = fmaf(y, y, sq), sk = fmaf(x, x, sk);
    if (threadIdx.x < 64) xq[c] = y, xk[c] = x, v[c] = w, num[c] = 0.f;
  }
  if (threadIdx.x == 0) v[d] = 1.f, num[d] = 0.f;
  fetch(4 * lane, 0);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sq += __shfl_xor(sq, o), sk += __shfl_xor(sk, o);
  __syncthreads();
  for (int l = threadIdx.x; l < M4; l += 256) {
    float p = 0.f, q = 0.f;
    if (l < M) {
      if constexpr (ELU) {
        p = xk[l], q = xq[l];
      } else {
        const float* __restrict__ w = a.W + (static_cast<size_t>(h) * M + l) * d;
        if (d % 4 == 0) {
#pragma unroll 4
          for (int c = 0; c < d; c += 4) {
            const float4 g = *reinterpret_cast<const float4*>(w + c);
            const float4 x = *reinterpret_cast<const float4*>(xk + c), y = *reinterpret_cast<const float4*>(xq + c);
            p = fmaf(g.x, x.x, p), p = fmaf(g.y, x.y, p), p = fmaf(g.z, x.z, p), p = fmaf(g.w, x.w, p);
            q = fmaf(g.x, y.x, q), q = fmaf(g.y, y.y, q), q = fmaf(g.z, y.z, q), q = fmaf(g.w, y.w, q);
          }
        } else {
          for (int c = 0; c < d; ++c) p = fmaf(w[c], xk[c], p), q = fmaf(w[c], xq[c], q);
        }
      }
    }
    auto phi = [&](float s, float square) {
      const bool nz = square > 0.f;
      if (a.nprf) s *= nz ? rsqrtf(square) : 0.f;
      if constexpr (ELU) return s > 0.f ? s + 1.f : expf(s);
      return expf(s - (a.nprf ? (nz ? 0.5f : 0.f) : 0.5f * square) + a.log_m);
    };
    fk[l] = l < M ? phi(p, sk) : 0.f;
    fq[l] = l < M ? phi(q, sq) : 0.f;
  }
  slot = check_slot(a.slots, slot, b, a.B);
  const float w = decay(rate_log2(a.rate[h]), 1);
  __syncthreads();
  for (int l0 = 0; l0 < M4; l0 += 4 * L) {  // (all lanes go round together)
    const int l = l0 + 4 * lane;
    float4 gq = make_float4(0.f, 0.f, 0.f, 0.f), gk = gq;
    if (l < M) gq = *reinterpret_cast<const float4*>(fq + l), gk = *reinterpret_cast<const float4*>(fk + l);
    for (int p = 0; p * K * R <= d; ++p) {
      if (p || l0) fetch(l, p);
      float s[K];
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const int c = (p * K + i) * R + r0;
        const float y = c <= d ? v[c] : 0.f;
        u[i].x = fmaf(w, u[i].x, y * gk.x), u[i].y = fmaf(w, u[i].y, y * gk.y);
        u[i].z = fmaf(w, u[i].z, y * gk.z), u[i].w = fmaf(w, u[i].w, y * gk.w);
        if (slot >= 0) store_cells<NT>(st, c, l, vec, u[i]);
        s[i] = fmaf(u[i].x, gq.x, fmaf(u[i].y, gq.y, fmaf(u[i].z, gq.z, u[i].w * gq.w)));
      }
      // lane bit by lane bit, the half of the rows that stays takes the other lane's parts
      int n = K, mine = 0;
#pragma unroll
      for (int o = L / 2; o >= 1; o >>= 1) {
        if (n > 1) {
          n >>= 1;
          const bool up = lane & o;
#pragma unroll
          for (int i = 0; i < K / 2; ++i)
            if (i < n) {
              const float keep = up ? s[i + n] : s[i], send = up ? s[i] : s[i + n];
              s[i] = keep + __shfl_xor(send, o);
            }
          mine += up ? n : 0;
        } else {
          s[0] += __shfl_xor(s[0], o);
        }
      }
      constexpr int spare = L > K ? L / K - 1 : 0;  // lanes that ended with the same row
      if (!(lane & spare))
#pragma unroll
        for (int i = 0; i < K; ++i)
          if (i < n) {
            const int c = (p * K + mine + i) * R + r0;
            if (c <= d) num[c] += s[i];
          }
    }
  }
  __syncthreads();
  TX* __restrict__ z = static_cast<TX*>(a.z) + row;
  const float inv = slot == kStateBad ? NAN : 1.f / num[d];
  for (int c = threadIdx.x; c < d; c += 256) {
    const float o = num[c] * inv;
    if constexpr (std::is_same<TX, float>::value)
      z[c] = o;
    else
      z[c] = static_cast<uint16_t>(pack_bf16(floatx2{o, 0.f}));
  }
}

// state[dst[i]] = state[src[i]] for all i at once (-1: zeros).  A thread owns the same cells of
// every slot: it reads them all into registers before it writes any, in the moves' order, so
// moves may overlap in any way and a slot written twice keeps the last.  CAP moves of a T fill
// up to 448 of a wave's 512 registers: that many reads are in flight, and one wave per SIMD
// fills HBM (the kept cells in LDS, read one by one: 106 us for 96 moves of 1 MiB; in registers:
// 41 us, 5.0 TB/s, a plain copy's rate).
template <typename T, int CAP>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(1))) void k_state_copy(
    T* __restrict__ state, const int* __restrict__ src, const int* __restrict__ dst, int count, int nslots, long long cells) {
  __shared__ int from[CAP], to[CAP];  // from -2: no move
  const long long e = static_cast<long long>(xcd_block(blockIdx.x, gridDim.x)) * 64 + threadIdx.x;
  for (int i = threadIdx.x; i < CAP; i += 64) {
    const int s = i < count ? src[i] : -2, t = i < count ? dst[i] : -1;
    from[i] = t >= 0 && t < nslots && s >= -1 && s < nslots ? s : -2;
    to[i] = t;
  }
  __syncthreads();
  const bool live = e < cells;
  T kept[CAP];
#pragma unroll
  for (int i = 0; i < CAP; ++i) {
    const int s = __builtin_amdgcn_readfirstlane(from[i]);
    kept[i] = T{};
    if (s >= 0 && live) kept[i] = state[s * cells + e];
  }
#pragma unroll
  for (int i = 0; i < CAP; ++i) {
    const int s = __builtin_amdgcn_readfirstlane(from[i]), t = __builtin_amdgcn_readfirstlane(to[i]);
    if (s >= -1 && live) state[t * cells + e] = kept[i];
  }
}

namespace {
template <typename TX, bool ELU>
void step(const PoolArgs& a, hipStream_t st) {
  const int M4 = (a.M + 3) & ~3, d4 = (a.d + 3) & ~3;
  const dim3 grid(static_cast<unsigned>(a.B) * a.H), block(256);
  const size_t lds = (4 * d4 + 2 * M4 + 8) * sizeof(float);
  // States that the last-level cache of 256 MiB does not hold go past it.  16 heads, 256 features,
  // d = 64, us with and without: 512 sequences (545 MB) 221 and 236; 256 (273 MB) 129 and 135 from memory,
  // 117 and 108 where the call before left part of them in the cache; 192 (204 MB) 90 and 69.
  const bool past = static_cast<size_t>(a.B) * a.H * (a.d + 1) * a.M * sizeof(float) > (size_t{256} << 20);
  auto go = [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    if (past)
      hipLaunchKernelGGL((k_decay_step<TX, L, ELU, true>), grid, block, lds, st, a);
    else
      hipLaunchKernelGGL((k_decay_step<TX, L, ELU, false>), grid, block, lds, st, a);
  };
  if (M4 <= 32)
    go(std::integral_constant<int, 8>{});
  else if (M4 <= 64)
    go(std::integral_constant<int, 16>{});
  else if (M4 <= 128)
    go(std::integral_constant<int, 32>{});
  else
    go(std::integral_constant<int, 64>{});
}
}  // namespace

hipError_t launch_decay_step(bool bf16, bool elu, const PoolArgs& a, hipStream_t st) {
  if (bf16)
    elu ? step<uint16_t, true>(a, st) : step<uint16_t, false>(a, st);
  else
    elu ? step<float, true>(a, st) : step<float, false>(a, st);
  return hipGetLastError();
}

namespace {
template <typename T, int CAP>
void copy_cells(float* state, const int* src, const int* dst, int count, int nslots, long long cells, hipStream_t st) {
  cells = cells * sizeof(float) / sizeof(T);
  hipLaunchKernelGGL((k_state_copy<T, CAP>), dim3(static_cast<unsigned>((cells + 63) / 64)), dim3(64), 0, st,
                     reinterpret_cast<T*>(state), src, dst, count, nslots, cells);
}
}  // namespace

hipError_t launch_state_copy(float* state, const int* src, const int* dst, int count, int nslots, long long cells,
                             hipStream_t st) {
  // the widest cells that the registers hold for so many moves
  if (cells % 4 == 0 && count <= 16)
    copy_cells<float4, 16>(state, src, dst, count, nslots, cells, st);
  else if (cells % 4 == 0 && count <= 64)
    copy_cells<float4, 64>(state, src, dst, count, nslots, cells, st);
  else if (cells % 4 == 0 && count <= 112)
    copy_cells<float4, 112>(state, src, dst, count, nslots, cells, st);
  else if (cells % 2 == 0 && count <= 224)
    copy_cells<float2, 224>(state, src, dst, count, nslots, cells, st);
  else
    copy_cells<float, 256>(state, src, dst, count, nslots, cells, st);
  return hipGetLastError();
}

}  // namespace krpe
