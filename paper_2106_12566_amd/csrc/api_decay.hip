// C ABI of attention with a decaying bias (declared in include/krpe.h): argument
// validation on the host, workspace carving and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "api_util.hpp"
#include "decay.hpp"
#include "krpe.h"

namespace krpe {
namespace {

int chunks(int n) { return static_cast<int>((static_cast<long long>(n) + kChunk - 1) / kChunk); }

// A prompt's sums: chunks of 128 positions in nseg segments of segc chunks.
struct DecayLayout {
  int nchunk, nseg, segc, Mp;
  size_t tot, pre, total;  // byte offsets
};

DecayLayout decay_layout(long long BH, int n, int d, int m, size_t off) {
  DecayLayout L{};
  L.Mp = (m + 31) & ~31;
  L.nchunk = chunks(n);
  // The number of segments from the rounds of work-groups that the sums take: a group of 128
  // features and a segment each, two to a CU (one beyond 64 dimensions, twice as many of the
  // two-wave groups of up to 64 features), a chunk costing one unit, a group's start a half and
  // the state of a segment, written and joined, a twentieth.  (16 heads of 256 features, 128 chunks: 22
  // segments, in two rounds, 117 us, 16 in one 85; 8 x 12 heads, 32 chunks: 8 in two rounds 127, 5 in one 131.)
  const long long groups = BH * ((L.Mp + 127) / 128);
  const long long slots = (d <= 64 ? 512 : 256) * (L.Mp <= 64 ? 2 : 1);
  double best = 0.0;
  L.nseg = 1, L.segc = L.nchunk > 1 ? L.nchunk : 1;
  for (int most = 1; most <= 256 && most <= L.nchunk; ++most) {
    const int segc = (L.nchunk + most - 1) / most, nseg = (L.nchunk + segc - 1) / segc;
    const double cost = static_cast<double>((groups * nseg + slots - 1) / slots) * (segc + 0.5) + 0.05 * nseg;
    if (most == 1 || cost < best) best = cost, L.nseg = nseg, L.segc = segc;
  }
  const size_t cells = static_cast<size_t>(d + 1) * L.Mp * sizeof(float);
  L.tot = off;
  L.pre = align_up(L.tot + BH * L.nseg * cells);
  L.total = align_up(L.pre + BH * L.nchunk * cells);
  return L;
}

struct BwdOffsets {
  DecayLayout f;
  size_t totb, preb, g, gd, total;
};
BwdOffsets bwd_offsets(long long BH, int n, int d, int m) {
  BwdOffsets o{};
  o.f = decay_layout(BH, n, d, m, 0);
  const DecayLayout r = decay_layout(BH, n, d, m, o.f.total);
  o.totb = r.tot, o.preb = r.pre;
  o.g = r.total;
  o.gd = align_up(o.g + static_cast<size_t>(BH) * n * d * sizeof(float));
  o.total = align_up(o.gd + static_cast<size_t>(BH) * n * sizeof(float));
  return o;
}

krpe_status_t check_sizes(int B, int H, int n, int d, int m, unsigned flags, unsigned known) {
  if (B < 0 || H < 0 || n < 0 || d < 0 || m < 0) return fail(KRPE_ERR_SHAPE, "negative size");
  if (flags & ~known) return fail(KRPE_ERR_UNSUPPORTED, "a flag bit that this call does not take");
  if (d < 1 || m < 1) return fail(KRPE_ERR_SHAPE, "d and m must be >= 1");
  if (d > kMaxD) return fail(KRPE_ERR_UNSUPPORTED, "d > 128 is not supported");
  if (m > kMaxM) return fail(KRPE_ERR_UNSUPPORTED, "m > 1024 is not supported");
  if ((flags & KRPE_FEAT_ELU) && m != d) return fail(KRPE_ERR_SHAPE, "KRPE_FEAT_ELU needs m == d");
  const long long bh = static_cast<long long>(B) * H;
  if (bh >= (1LL << 31) || (n > 0 && bh > ((1LL << 31) - 1) / n))
    return fail(KRPE_ERR_UNSUPPORTED, "B * H * n >= 2^31 is not supported");
  // (a grid of 256-thread groups, one for each head's chunk)
  if (bh * std::max(1, chunks(n)) >= (1LL << 24))
    return fail(KRPE_ERR_UNSUPPORTED, "2^24 or more chunks of 128 positions are not supported");
  return KRPE_OK;
}
krpe_status_t check_dtype(int dt) {
  return dt == KRPE_F32 || dt == KRPE_BF16 ? KRPE_OK : fail(KRPE_ERR_DTYPE, "qkv_dtype must be F32 or BF16");
}
bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

constexpr unsigned kFlags = KRPE_NPRF | KRPE_FEAT_ELU;

size_t state_bytes(int slots, int H, int d, int m) {
  return static_cast<size_t>(slots) * H * (d + 1) * m * sizeof(float);
}
size_t weight_bytes(int H, int d, int m, unsigned flags) {
  return flags & KRPE_FEAT_ELU ? 0 : static_cast<size_t>(H) * m * d * sizeof(float);
}

// What a pool's calls share; rows: tokens of a sequence in q, k, v.
krpe_status_t check_pool(int dt, const float* rate, const float* W, const float* state, const int* slots, int nslots,
                         int B, int H, int rows, int d, int m, unsigned flags) {
  if (krpe_status_t s = check_sizes(B, H, rows, d, m, flags, kFlags)) return s;
  if (krpe_status_t s = check_dtype(dt)) return s;
  if (nslots < 0 || (!slots && nslots < B)) return fail(KRPE_ERR_SHAPE, "the pool needs a slot for each sequence");
  if (static_cast<long long>(B) * H * rows == 0) return KRPE_OK;
  if (!rate || (!(flags & KRPE_FEAT_ELU) && !W) || !state)
    return fail(KRPE_ERR_NULL, "rate, W (but for elu + 1) and state must be non-NULL");
  if (misaligned(state) || misaligned(W) || off4(rate) || off4(slots))
    return fail(KRPE_ERR_ALIGN, "pointers must be 16-byte aligned (rate and integers 4)");
  return KRPE_OK;
}

PoolArgs pool_args(const void* q, const void* k, const void* v, void* z, const float* rate, const float* W, float* state,
                   const int* slots, int nslots, int B, int H, int d, int m, unsigned flags) {
  PoolArgs a{};
  a.q = q, a.k = k, a.v = v, a.z = z, a.rate = rate, a.W = W, a.state = state, a.slots = slots;
  a.B = B, a.H = H, a.d = d, a.M = m, a.nslots = nslots, a.nprf = (flags & KRPE_NPRF) != 0;
  a.log2_m = -0.5 * std::log2(static_cast<double>(m));
  a.log_m = static_cast<float>(-0.5 * std::log(static_cast<double>(m)));
  return a;
}

}  // namespace
}  // namespace krpe

using namespace krpe;

extern "C" {

size_t krpe_decay_fwd_workspace(int B, int H, int n, int d, int m, unsigned flags) {
  if (check_sizes(B, H, n, d, m, flags, kFlags | KRPE_STATE_FRESH | KRPE_ZERO_TAIL) != KRPE_OK) return 0;
  return decay_layout(static_cast<long long>(B) * H, n, d, m, 0).total;
}

krpe_status_t krpe_decay_fwd(const void* q, const void* k, const void* v, int qkv_dtype, const float* rate,
                             const float* W, void* z, float* state, const int* slots, int nslots, const int* lens,
                             int B, int H, int n, int d, int m, unsigned flags, void* ws, size_t ws_bytes,
                             void* stream) {
  clear_error();
  if (krpe_status_t s = check_sizes(B, H, n, d, m, flags, kFlags | KRPE_STATE_FRESH | KRPE_ZERO_TAIL)) return s;
  if (krpe_status_t s = check_dtype(qkv_dtype)) return s;
  if (!state && (slots || nslots)) return fail(KRPE_ERR_NULL, "slots without a pool of states");
  if (!state && (flags & KRPE_STATE_FRESH)) return fail(KRPE_ERR_NULL, "KRPE_STATE_FRESH without a pool of states");
  if (nslots < 0 || (state && !slots && nslots < B)) return fail(KRPE_ERR_SHAPE, "the pool needs a slot for each sequence");
  const long long bh = static_cast<long long>(B) * H;
  if (bh == 0 || (n == 0 && !state)) return KRPE_OK;
  const bool elu = (flags & KRPE_FEAT_ELU) != 0;
  if (!rate || (!elu && !W) || (n > 0 && (!q || !k || !v || !z)))
    return fail(KRPE_ERR_NULL, "q, k, v, rate, W (but for elu + 1) and z must be non-NULL");
  const void* ptrs[] = {q, k, v, z, W, state, ws};
  for (const void* p : ptrs)
    if (misaligned(p)) return fail(KRPE_ERR_ALIGN, "pointers must be 16-byte aligned (rate and integers 4)");
  if (off4(rate) || off4(slots) || off4(lens))
    return fail(KRPE_ERR_ALIGN, "pointers must be 16-byte aligned (rate and integers 4)");
  const DecayLayout L = decay_layout(bh, n, d, m, 0);
  if (!ws || ws_bytes < L.total) return fail(KRPE_ERR_WORKSPACE, "workspace needs " + std::to_string(L.total) + " bytes");
  const size_t x = static_cast<size_t>(bh) * n * d * dtype_size(qkv_dtype);
  const Range ins[] = {{q, x}, {k, x}, {v, x}, {rate, H * sizeof(float)}, {W, weight_bytes(H, d, m, flags)},
                       {slots, slots ? B * sizeof(int) : 0}, {lens, lens ? B * sizeof(int) : 0}};
  const Range outs[] = {{z, x}, {state, state ? state_bytes(nslots, H, d, m) : 0}, {ws, ws_bytes}};
  for (int o = 0; o < 3; ++o) {
    for (const Range& r : ins)
      if (overlaps(outs[o], r)) return fail(KRPE_ERR_ALIAS, "an output or the workspace overlaps an input");
    for (int p = o + 1; p < 3; ++p)
      if (overlaps(outs[o], outs[p])) return fail(KRPE_ERR_ALIAS, "outputs overlap each other or the workspace");
  }
  char* w = static_cast<char*>(ws);
  DecayArgs a{};
  a.q = q, a.k = k, a.v = v, a.z = z, a.rate = rate, a.W = W, a.state = state, a.slots = slots, a.lens = lens;
  a.tot = reinterpret_cast<float*>(w + L.tot);
  a.pre = reinterpret_cast<float*>(w + L.pre);
  a.B = B, a.H = H, a.n = n, a.d = d, a.M = m, a.Mp = L.Mp, a.nchunk = L.nchunk, a.nseg = L.nseg, a.segc = L.segc;
  a.nslots = nslots, a.nprf = (flags & KRPE_NPRF) != 0, a.fresh = (flags & KRPE_STATE_FRESH) != 0;
  a.tail = lens && (flags & KRPE_ZERO_TAIL);
  a.log2_m = -0.5 * std::log2(static_cast<double>(m));
  return hip_check(launch_decay_fwd(qkv_dtype == KRPE_BF16, elu, a, static_cast<hipStream_t>(stream)), "decay launch");
}

size_t krpe_decay_bwd_workspace(int B, int H, int n, int d, int m, unsigned flags) {
  if (check_sizes(B, H, n, d, m, flags, kFlags | KRPE_ZERO_TAIL) != KRPE_OK) return 0;
  return bwd_offsets(static_cast<long long>(B) * H, n, d, m).total;
}

krpe_status_t krpe_decay_bwd(const void* q, const void* k, const void* v, int qkv_dtype, const float* rate,
                             const float* W, const void* dz, void* dq, void* dk, void* dv, const int* lens, int B,
                             int H, int n, int d, int m, unsigned flags, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  if (krpe_status_t s = check_sizes(B, H, n, d, m, flags, kFlags | KRPE_ZERO_TAIL)) return s;
  if (krpe_status_t s = check_dtype(qkv_dtype)) return s;
  const long long bh = static_cast<long long>(B) * H;
  if (bh * n == 0) return KRPE_OK;
  const bool elu = (flags & KRPE_FEAT_ELU) != 0;
  if (!q || !k || !v || !rate || (!elu && !W) || !dz || !dq || !dk || !dv)
    return fail(KRPE_ERR_NULL, "q, k, v, rate, W (but for elu + 1), dz, dq, dk and dv must be non-NULL");
  const void* ptrs[] = {q, k, v, W, dz, dq, dk, dv, ws};
  for (const void* p : ptrs)
    if (misaligned(p)) return fail(KRPE_ERR_ALIGN, "pointers must be 16-byte aligned (rate and integers 4)");
  if (off4(rate) || off4(lens)) return fail(KRPE_ERR_ALIGN, "pointers must be 16-byte aligned (rate and integers 4)");
  const BwdOffsets o = bwd_offsets(bh, n, d, m);
  if (!ws || ws_bytes < o.total) return fail(KRPE_ERR_WORKSPACE, "workspace needs " + std::to_string(o.total) + " bytes");
  const size_t x = static_cast<size_t>(bh) * n * d * dtype_size(qkv_dtype);
  const Range ins[] = {{q, x}, {k, x}, {v, x}, {dz, x}, {rate, H * sizeof(float)}, {W, weight_bytes(H, d, m, flags)},
                       {lens, lens ? B * sizeof(int) : 0}};
  const Range outs[] = {{dq, x}, {dk, x}, {dv, x}, {ws, ws_bytes}};
  for (int p = 0; p < 4; ++p) {
    for (const Range& r : ins)
      if (overlaps(outs[p], r)) return fail(KRPE_ERR_ALIAS, "an output or the workspace overlaps an input");
    for (int p2 = p + 1; p2 < 4; ++p2)
      if (overlaps(outs[p], outs[p2])) return fail(KRPE_ERR_ALIAS, "outputs overlap each other or the workspace");
  }
  char* w = static_cast<char*>(ws);
  DecayArgs a{};
  a.q = q, a.k = k, a.v = v, a.rate = rate, a.W = W, a.lens = lens, a.dz = dz, a.dq = dq, a.dk = dk, a.dv = dv;
  a.tot = reinterpret_cast<float*>(w + o.f.tot), a.pre = reinterpret_cast<float*>(w + o.f.pre);
  a.totb = reinterpret_cast<float*>(w + o.totb), a.preb = reinterpret_cast<float*>(w + o.preb);
  a.g = reinterpret_cast<float*>(w + o.g), a.gd = reinterpret_cast<float*>(w + o.gd);
  a.B = B, a.H = H, a.n = n, a.d = d, a.M = m, a.Mp = o.f.Mp, a.nchunk = o.f.nchunk, a.nseg = o.f.nseg, a.segc = o.f.segc;
  a.nprf = (flags & KRPE_NPRF) != 0, a.tail = lens && (flags & KRPE_ZERO_TAIL);
  a.log2_m = -0.5 * std::log2(static_cast<double>(m));
  return hip_check(launch_decay_bwd(qkv_dtype == KRPE_BF16, elu, a, static_cast<hipStream_t>(stream)),
                   "decay backward launch");
}

krpe_status_t krpe_decay_step(const void* q, const void* k, const void* v, int qkv_dtype, const float* rate,
                              const float* W, void* z, float* state, const int* slots, int nslots, int B, int H, int d,
                              int m, unsigned flags, void* stream) {
  clear_error();
  if (krpe_status_t s = check_pool(qkv_dtype, rate, W, state, slots, nslots, B, H, 1, d, m, flags)) return s;
  const long long bh = static_cast<long long>(B) * H;
  if (bh == 0) return KRPE_OK;
  if (!q || !k || !v || !z) return fail(KRPE_ERR_NULL, "q, k, v and z must be non-NULL");
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(z))
    return fail(KRPE_ERR_ALIGN, "pointers must be 16-byte aligned (rate and integers 4)");
  const size_t x = static_cast<size_t>(bh) * d * dtype_size(qkv_dtype);
  const Range ins[] = {{q, x}, {k, x}, {v, x}, {rate, H * sizeof(float)}, {W, weight_bytes(H, d, m, flags)},
                       {slots, slots ? B * sizeof(int) : 0}};
  const Range rz{z, x}, rs{state, state_bytes(nslots, H, d, m)};
  for (const Range& r : ins)
    if (overlaps(rz, r) || overlaps(rs, r)) return fail(KRPE_ERR_ALIAS, "z or the states overlap an input");
  if (overlaps(rz, rs)) return fail(KRPE_ERR_ALIAS, "z overlaps the states");
  const PoolArgs a = pool_args(q, k, v, z, rate, W, state, slots, nslots, B, H, d, m, flags);
  return hip_check(launch_decay_step(qkv_dtype == KRPE_BF16, (flags & KRPE_FEAT_ELU) != 0, a,
                                     static_cast<hipStream_t>(stream)),
                   "decay step launch");
}

krpe_status_t krpe_decay_tree(const void* q, const void* k, const void* v, int qkv_dtype, const int* parent,
                              const float* rate, const float* W, void* z, const float* state, const int* slots,
                              int nslots, int B, int H, int T, int d, int m, unsigned flags, void* stream) {
  clear_error();
  if (krpe_status_t s = check_pool(qkv_dtype, rate, W, state, slots, nslots, B, H, T, d, m, flags)) return s;
  if (T > KRPE_TREE_MAX) return fail(KRPE_ERR_UNSUPPORTED, "a tree of more than 64 nodes is not supported");
  const long long bh = static_cast<long long>(B) * H;
  if (bh * T == 0) return KRPE_OK;
  if (!q || !k || !v || !z || !parent) return fail(KRPE_ERR_NULL, "q, k, v, z and parent must be non-NULL");
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(z) || off4(parent))
    return fail(KRPE_ERR_ALIGN, "pointers must be 16-byte aligned (rate and integers 4)");
  const size_t x = static_cast<size_t>(bh) * T * d * dtype_size(qkv_dtype);
  const Range ins[] = {{q, x}, {k, x}, {v, x}, {rate, H * sizeof(float)}, {W, weight_bytes(H, d, m, flags)},
                       {slots, slots ? B * sizeof(int) : 0}, {parent, static_cast<size_t>(B) * T * sizeof(int)},
                       {state, state_bytes(nslots, H, d, m)}};
  for (const Range& r : ins)
    if (overlaps({z, x}, r)) return fail(KRPE_ERR_ALIAS, "z overlaps an input or the states");
  PoolArgs a = pool_args(q, k, v, z, rate, W, const_cast<float*>(state), slots, nslots, B, H, d, m, flags);
  a.parent = parent, a.T = T;
  return hip_check(launch_decay_tree(qkv_dtype == KRPE_BF16, (flags & KRPE_FEAT_ELU) != 0, a,
                                     static_cast<hipStream_t>(stream)),
                   "decay tree launch");
}

krpe_status_t krpe_decay_commit(const void* k, const void* v, int qkv_dtype, const int* path, const float* rate,
                                const float* W, float* state, const int* slots, int nslots, int B, int H, int T, int P,
                                int d, int m, unsigned flags, void* stream) {
  clear_error();
  if (krpe_status_t s = check_pool(qkv_dtype, rate, W, state, slots, nslots, B, H, T, d, m, flags)) return s;
  if (P < 0) return fail(KRPE_ERR_SHAPE, "negative size");
  if (T > 65536) return fail(KRPE_ERR_UNSUPPORTED, "more than 65536 tokens to choose from is not supported");
  if (P >= 1 << 30) return fail(KRPE_ERR_UNSUPPORTED, "a path of 2^30 or more entries is not supported");
  const long long bh = static_cast<long long>(B) * H;
  if (bh * T == 0 || P == 0) return KRPE_OK;
  if (!k || !v || !path) return fail(KRPE_ERR_NULL, "k, v and path must be non-NULL");
  if (misaligned(k) || misaligned(v) || off4(path))
    return fail(KRPE_ERR_ALIGN, "pointers must be 16-byte aligned (rate and integers 4)");
  const size_t x = static_cast<size_t>(bh) * T * d * dtype_size(qkv_dtype);
  const Range ins[] = {{k, x}, {v, x}, {rate, H * sizeof(float)}, {W, weight_bytes(H, d, m, flags)},
                       {slots, slots ? B * sizeof(int) : 0}, {path, static_cast<size_t>(B) * P * sizeof(int)}};
  for (const Range& r : ins)
    if (overlaps({state, state_bytes(nslots, H, d, m)}, r)) return fail(KRPE_ERR_ALIAS, "the states overlap an input");
  DecayArgs a{};
  a.k = k, a.v = v, a.rate = rate, a.W = W, a.state = state, a.slots = slots, a.path = path;
  a.B = B, a.H = H, a.n = T, a.P = P, a.d = d, a.M = m, a.Mp = (m + 31) & ~31, a.nseg = 1;
  a.nslots = nslots, a.nprf = (flags & KRPE_NPRF) != 0;
  a.log2_m = -0.5 * std::log2(static_cast<double>(m));
  return hip_check(launch_decay_commit(qkv_dtype == KRPE_BF16, (flags & KRPE_FEAT_ELU) != 0, a,
                                       static_cast<hipStream_t>(stream)),
                   "decay commit launch");
}

krpe_status_t krpe_decay_state_copy(float* state, const int* src, const int* dst, int count, int nslots, int H, int d,
                                    int m, void* stream) {
  clear_error();
  if (krpe_status_t s = check_sizes(1, 1, 0, d, m, 0u, 0u)) return s;
  if (nslots < 0 || H < 0 || count < 0) return fail(KRPE_ERR_SHAPE, "negative size");
  if (static_cast<long long>(H) * (d + 1) * m >= (1LL << 31))
    return fail(KRPE_ERR_UNSUPPORTED, "a slot of 2^31 or more elements is not supported");
  if (count > KRPE_COPY_MAX) return fail(KRPE_ERR_UNSUPPORTED, "more than 256 moves in a call are not supported");
  if (count == 0 || nslots == 0 || H == 0) return KRPE_OK;
  if (!state || !src || !dst) return fail(KRPE_ERR_NULL, "state, src and dst must be non-NULL");
  if (misaligned(state) || off4(src) || off4(dst))
    return fail(KRPE_ERR_ALIGN, "pointers must be 16-byte aligned (rate and integers 4)");
  const Range rs{state, state_bytes(nslots, H, d, m)};
  if (overlaps(rs, {src, count * sizeof(int)}) || overlaps(rs, {dst, count * sizeof(int)}))
    return fail(KRPE_ERR_ALIAS, "the states overlap src or dst");
  return hip_check(launch_state_copy(state, src, dst, count, nslots, static_cast<long long>(H) * (d + 1) * m,
                                     static_cast<hipStream_t>(stream)),
                   "state copy launch");
}

}  // extern "C"
