// gfx950 (MI355X) rotary positions with several axes on queries and keys.
//
// The d = 64 features of a head form 32 pairs; pair i belongs to one axis a(i)
// (time, height, width, sensor, ...) and is turned as a complex number by the
// angle pos_{a(i)} f_i.  Pairs behind the last axis' are copied.  The turn by
// the negative angle undoes it and is its gradient.
//
// Bound by HBM: Q and K are read and written once (4 bytes per bf16 value).
// The angle is formed in fp64 as turns (pos f / 2 pi, f on the host), and its
// fraction is exact however far the position, so only the sine and cosine of
// an angle of at most half a turn are fp32.  They depend on the token and pair
// alone: a thread forms them once for eight pairs of a token and turns the
// pairs of many heads with them.
#include <hip/hip_runtime.h>

#include <float.h>
#include <stdint.h>

#include "ga_internal.h"

namespace ga {
namespace {

#include "ga_device.h"

// A thread takes 16 bytes of a row, so that a wave's loads are whole rows
// (107 us at B H = 128, n = 8000 against 110 with two loads of half rows, both
// through the caches).
// Interleaved, its values are pairs; in the halves' layout they are one side of
// as many pairs, whose other side the mirrored thread of the row holds: thread s
// of T has values kPer s of the first half, thread T - 1 - s those of the second.
template <class DT, bool INTERLEAVED>
struct Tile {
  static constexpr int kPer = 128 / DT::kBits;  // values in 16 bytes
  static constexpr int kPairs = INTERLEAVED ? kPer / 2 : kPer;
  static constexpr int kThreads = 64 / kPer;      // threads per token: 8 (bf16) or 16
  static constexpr int kTokens = 256 / kThreads;  // tokens per workgroup
  u32x4 w;

  static __device__ __forceinline__ bool second(int s) { return !INTERLEAVED && s >= kThreads / 2; }
  static __device__ __forceinline__ int pair0(int s) { return kPairs * (second(s) ? kThreads - 1 - s : s); }
  static __device__ __forceinline__ int offset(int s) {
    return INTERLEAVED ? kPer * s : pair0(s) + (second(s) ? 32 : 0);
  }
  __device__ __forceinline__ void load(const typename DT::T* p) { w = *(const u32x4*)p; }
  static __device__ __forceinline__ float value(const u32x4& w, int e) {
    if constexpr (DT::kBits == 16)
      return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    else
      return __uint_as_float(w[e]);
  }
  // halves: si is negated in the first half's threads; same: the pair stays as it
  // is, whatever it holds (zero times infinity is not zero)
  template <bool PAST>
  __device__ __forceinline__ void turn(const float (&co)[kPairs], const float (&si)[kPairs],
                                       const bool (&same)[kPairs], typename DT::T* p) const {
    float v[kPer];
    if constexpr (INTERLEAVED) {
#pragma unroll
      for (int m = 0; m < kPairs; ++m) {
        const float a = value(w, 2 * m), c = value(w, 2 * m + 1);
        v[2 * m] = same[m] ? a : a * co[m] - c * si[m];
        v[2 * m + 1] = same[m] ? c : c * co[m] + a * si[m];
      }
    } else {
      u32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (uint32_t)dpp<kThreads == 8 ? kHalfMirror : kMirror>((int)w[e]);
#pragma unroll
      for (int m = 0; m < kPairs; ++m) v[m] = same[m] ? value(w, m) : value(w, m) * co[m] + value(o, m) * si[m];
    }
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (DT::kBits == 16)
        o[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
      else
        o[e] = __float_as_uint(v[e]);
    }
    if constexpr (PAST)
      __builtin_nontemporal_store(o, (u32x4*)p);
    else
      *(u32x4*)p = o;
  }
};

// grid (ceil(n / kTokens), head shares, B).  Workgroup y takes heads y, y + gridDim.y, ...
// of the H query heads followed by the Hk key heads.  PAST: the outputs are
// written past the caches.
template <class DT, bool INTERLEAVED, bool PAST>
__global__ __launch_bounds__(256) void k_rotary(const typename DT::T* Q, const typename DT::T* K, const void* pos,
                                                RotaryPlan P, int H, int Hk, int n, typename DT::T* Qo,
                                                typename DT::T* Ko) {
  using R = Tile<DT, INTERLEAVED>;
  const int t = blockIdx.x * R::kTokens + threadIdx.x / R::kThreads, s = threadIdx.x % R::kThreads;
  if (t >= n) return;
  const int64_t b = blockIdx.z, pb = P.pos_batches > 1 ? b : 0;
  // a head's row is requested two heads before its turn is written, the first
  // ones before the angles are formed
  auto row = [&](int h) __attribute__((always_inline)) {
    return ((h < H ? b * H + h : b * Hk + (h - H)) * n + t) * 64 + R::offset(s);
  };
  const int step = gridDim.y, heads = H + Hk;
  R x[2];
  auto request = [&](int h, R& to) __attribute__((always_inline)) {
    if (h < heads) to.load((h < H ? Q : K) + row(h));
  };
  request(blockIdx.y, x[0]);
  request(blockIdx.y + step, x[1]);
  float co[R::kPairs], si[R::kPairs];
  bool same[R::kPairs];
#pragma unroll
  for (int e = 0; e < R::kPairs; ++e) {
    const int i = R::pair0(s) + e;
    const int64_t at = ((int64_t)P.axis[i] * P.pos_batches + pb) * n + t;
    const double x = P.pos_float ? (double)((const float*)pos)[at] : (double)((const int32_t*)pos)[at];
    const double turns = x * P.turns[i];
    const float f = (float)(turns - rint(turns));  // [-1/2, 1/2]
    si[e] = __builtin_amdgcn_sinf(f);  // of f turns; off by at most 2^-23 there (measured over 2^22 values)
    co[e] = __builtin_amdgcn_cosf(f);
    if (!INTERLEAVED && !R::second(s)) si[e] = -si[e];
    same[e] = P.turns[i] == 0.0;
  }
  for (int h = blockIdx.y; h < heads; h += 2 * step) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int g = h + u * step;
      if (g >= heads) break;
      const R now = x[u];
      request(g + 2 * step, x[u]);
      now.template turn<PAST>(co, si, same, (g < H ? Qo : Ko) + row(g));
    }
  }
}

}  // namespace

hipError_t launch_rotary(int dtype, int B, int H, int Hk, int n, const void* Q, const void* K, const void* pos,
                         const RotaryPlan& plan, bool interleaved, void* Qo, void* Ko, hipStream_t st) {
  const int tokens = dtype == 1 ? (interleaved ? Tile<BF16, true>::kTokens : Tile<BF16, false>::kTokens)
                                : (interleaved ? Tile<F32, true>::kTokens : Tile<F32, false>::kTokens);
  const unsigned tiles = (unsigned)((n + tokens - 1) / tokens);
  const int heads = H + Hk;
  // the sines are formed once per workgroup, so a workgroup takes every head of
  // its tokens unless that leaves compute units idle
  const int64_t wgs = (int64_t)tiles * B;
  int64_t shares = (1024 + wgs - 1) / wgs;
  if (shares > heads) shares = heads;
  const dim3 grid(tiles, (unsigned)shares, (unsigned)B);
  // Outputs that the last-level cache (256 MiB) holds are left to it, for whoever
  // reads them next; more than three quarters of it would only drive each other
  // out.  With the attention that reads them, bf16, B H = 128, n = 8000 (262 MB):
  // 227 us past the caches and 231 through them, alone 103 and 107; B H = 64 (131
  // MB): 125 and 123.
  const bool past = (int64_t)B * heads * n * (dtype == 1 ? 128 : 256) > (192 << 20);
  TimedLaunch tl("rotary", st);
#define GA_ROT(DT, I, PAST)                                                                                      \
  hipLaunchKernelGGL((k_rotary<DT, I, PAST>), grid, dim3(256), 0, st, (const typename DT::T*)Q,                    \
                     (const typename DT::T*)K, pos, plan, H, Hk, n, (typename DT::T*)Qo, (typename DT::T*)Ko)
#define GA_ROT_PAST(DT, I)          \
  do {                              \
    if (past) GA_ROT(DT, I, true);  \
    else GA_ROT(DT, I, false);      \
  } while (0)
  if (dtype == 1) {
    if (interleaved) GA_ROT_PAST(BF16, true);
    else GA_ROT_PAST(BF16, false);
  } else {
    if (interleaved) GA_ROT_PAST(F32, true);
    else GA_ROT_PAST(F32, false);
  }
#undef GA_ROT_PAST
#undef GA_ROT
  return hipGetLastError();
}

}  // namespace ga
