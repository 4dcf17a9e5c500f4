// Single tokens (krpe_decay_step) and copies within a pool of states
// (krpe_decay_state_copy), both bound by the states' bytes.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "decay.hpp"

namespace krpe {

// Features of R rows x [R][d] in LDS (fp32), f [R][M4] (zeros from M to M4).  A group of 2^g
// lanes takes a feature, each a part of its dimensions.
template <int R, bool ELU>
__device__ __forceinline__ void row_features(const float* __restrict__ x, const float* __restrict__ sq,
                                             const float* __restrict__ W, int d, int M, int M4, float log_m, bool nprf,
                                             float* __restrict__ f) {
  for (int l = threadIdx.x; l < M4; l += blockDim.x) {
    float acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = 0.f;
    if (l < M) {
      if constexpr (ELU) {
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r] = x[r * d + l];
      } else {
        const float* __restrict__ w = W + static_cast<size_t>(l) * d;
        if (d % 4 == 0) {
          for (int c = 0; c < d; c += 4) {
            const float4 u = *reinterpret_cast<const float4*>(w + c);
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float4 y = *reinterpret_cast<const float4*>(x + r * d + c);
              acc[r] = fmaf(u.x, y.x, acc[r]), acc[r] = fmaf(u.y, y.y, acc[r]);
              acc[r] = fmaf(u.z, y.z, acc[r]), acc[r] = fmaf(u.w, y.w, acc[r]);
            }
          }
        } else {
          for (int c = 0; c < d; ++c)
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r] = fmaf(w[c], x[r * d + c], acc[r]);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float o = 0.f;
      if (l < M) {
        const float s = nprf ? (sq[r] > 0.f ? rsqrtf(sq[r]) : 0.f) : 1.f;
        if constexpr (ELU) {
          const float y = acc[r] * s;
          o = y > 0.f ? y + 1.f : expf(y);
        } else {
          const float half = nprf ? (sq[r] > 0.f ? 0.5f : 0.f) : 0.5f * sq[r];
          o = expf(acc[r] * s - half + log_m);
        }
      }
      f[r * M4 + l] = o;
    }
  }
}

// The sums of squares of R rows in LDS, one wave a row.
template <int R>
__device__ __forceinline__ void row_squares(const float* __restrict__ x, int d, float* __restrict__ sq) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  for (int r = wave; r < R; r += waves) {
    float s = 0.f;
    for (int c = lane; c < d; c += 64) s = fmaf(x[r * d + c], x[r * d + c], s);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o);
    if (lane == 0) sq[r] = s;
  }
}

// Lanes of a wave on one row of a state (a power of two), four features each.
__device__ __forceinline__ int lanes_of(int M4) {
  int n = 1;
  while (n < 64 && n * 4 < M4) n <<= 1;
  return n;
}
__device__ __forceinline__ float4 load_cells(const float* __restrict__ p, int l, int M, bool vec) {
  if (vec) return *reinterpret_cast<const float4*>(p + l);
  return make_float4(p[l], l + 1 < M ? p[l + 1] : 0.f, l + 2 < M ? p[l + 2] : 0.f, l + 3 < M ? p[l + 3] : 0.f);
}
__device__ __forceinline__ void store_cells(float* __restrict__ p, int l, int M, bool vec, float4 v) {
  if (vec) {
    *reinterpret_cast<float4*>(p + l) = v;
  } else {
    p[l] = v.x;
    if (l + 1 < M) p[l + 1] = v.y;
    if (l + 2 < M) p[l + 2] = v.z;
    if (l + 3 < M) p[l + 3] = v.w;
  }
}

// One token of a sequence and head: A <- e^-rate A + [v; 1] phi(k)^T, z = A phi(q).
template <typename TX, bool ELU>
__global__ __launch_bounds__(256) void k_decay_step(PoolArgs a) {
  extern __shared__ __align__(16) float sm[];
  const int d = a.d, M = a.M, M4 = (M + 3) & ~3, d4 = (d + 3) & ~3;
  float *x = sm, *f = sm + 2 * d4, *v = f + 2 * M4, *num = v + d + 1;  // num: d + 1 sums
  __shared__ float sq[2];
  const int b = blockIdx.x / a.H, h = blockIdx.x % a.H;
  const int slot = slot_of(a.slots, b, a.B, a.nslots);
  const size_t row = static_cast<size_t>(blockIdx.x) * d;
  for (int c = threadIdx.x; c < d; c += 256) {
    x[c] = to_f32(static_cast<const TX*>(a.q)[row + c]);
    x[d + c] = to_f32(static_cast<const TX*>(a.k)[row + c]);
    v[c] = to_f32(static_cast<const TX*>(a.v)[row + c]);
  }
  if (threadIdx.x == 0) v[d] = 1.f;
  __syncthreads();
  row_squares<2>(x, d, sq);
  __syncthreads();
  row_features<2, ELU>(x, sq, a.W + static_cast<size_t>(h) * M * d, d, M, M4, a.log_m, a.nprf, f);
  __syncthreads();
  const int L = lanes_of(M4), lane = threadIdx.x % L, per = 256 / L;
  const float w = decay(rate_log2(a.rate[h]), 1);
  const bool vec = M % 4 == 0;
  float* __restrict__ st = slot >= 0 ? a.state + (static_cast<size_t>(slot) * a.H + h) * (d + 1) * M : nullptr;
  for (int c0 = 0; c0 <= d; c0 += per) {
    const int c = c0 + threadIdx.x / L;
    float s = 0.f;
    if (c <= d)
      for (int l = 4 * lane; l < M; l += 4 * L) {
        const float4 fq = *reinterpret_cast<const float4*>(f + l), fk = *reinterpret_cast<const float4*>(f + M4 + l);
        float4 u = make_float4(0.f, 0.f, 0.f, 0.f);
        if (st) u = load_cells(st + static_cast<size_t>(c) * M, l, M, vec);
        u.x = fmaf(w, u.x, v[c] * fk.x), u.y = fmaf(w, u.y, v[c] * fk.y);
        u.z = fmaf(w, u.z, v[c] * fk.z), u.w = fmaf(w, u.w, v[c] * fk.w);
        if (st) store_cells(st + static_cast<size_t>(c) * M, l, M, vec, u);
        s = fmaf(u.x, fq.x, s), s = fmaf(u.y, fq.y, s), s = fmaf(u.z, fq.z, s), s = fmaf(u.w, fq.w, s);
      }
    for (int o = 1; o < L; o <<= 1) s += __shfl_xor(s, o);
    if (c <= d && lane == 0) num[c] = s;
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

hipError_t launch_decay_step(bool bf16, bool elu, const PoolArgs& a, hipStream_t st) {
  const int M4 = (a.M + 3) & ~3, d4 = (a.d + 3) & ~3;
  const dim3 grid(static_cast<unsigned>(a.B) * a.H), block(256);
  const size_t lds = (2 * d4 + 2 * M4 + 2 * (a.d + 1)) * sizeof(float);
  if (bf16)
    elu ? k_decay_step<uint16_t, true><<<grid, block, lds, st>>>(a) : k_decay_step<uint16_t, false><<<grid, block, lds, st>>>(a);
  else
    elu ? k_decay_step<float, true><<<grid, block, lds, st>>>(a) : k_decay_step<float, false><<<grid, block, lds, st>>>(a);
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
