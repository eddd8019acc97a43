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

constexpr int kTok = 64;  // tokens per workgroup: four threads each, eight pairs a thread

template <class DT>
struct Half8 {  // eight values as stored
  static constexpr int kWords = DT::kBits == 16 ? 1 : 2;
  u32x4 w[kWords];
  __device__ __forceinline__ void load(const typename DT::T* p) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = ((const u32x4*)p)[i];
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (DT::kBits == 16)
        v[e] = __uint_as_float(e & 1 ? w[0][e / 2] & 0xffff0000u : w[0][e / 2] << 16);
      else
        v[e] = __uint_as_float(w[e / 4][e % 4]);
    }
  }
  static __device__ __forceinline__ void store(typename DT::T* p, const float (&v)[8]) {
    if constexpr (DT::kBits == 16) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
      *(u32x4*)p = w;
    } else {
      *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
      *(float4*)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
};

// grid (ceil(n / 64), head shares, B).  Workgroup y takes heads y, y + gridDim.y, ...
// of the H query heads followed by the Hk key heads.
template <class DT, bool INTERLEAVED>
__global__ __launch_bounds__(256) void k_rotary(const typename DT::T* Q, const typename DT::T* K, const void* pos,
                                                RotaryPlan P, int H, int Hk, int n, typename DT::T* Qo,
                                                typename DT::T* Ko) {
  const int t = blockIdx.x * kTok + (threadIdx.x >> 2), s = threadIdx.x & 3;
  if (t >= n) return;
  const int64_t b = blockIdx.z, pb = P.pos_batches > 1 ? b : 0;
  float co[8], si[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = 8 * s + e;
    const int64_t at = ((int64_t)P.axis[i] * P.pos_batches + pb) * n + t;
    const double x = P.pos_float ? (double)((const float*)pos)[at] : (double)((const int32_t*)pos)[at];
    const double turns = x * P.turns[i];
    const float f = (float)(turns - rint(turns));  // [-1/2, 1/2]
    sincospif(2.0f * f, &si[e], &co[e]);
  }
  const int lo = INTERLEAVED ? 16 * s : 8 * s, hi = INTERLEAVED ? 16 * s + 8 : 32 + 8 * s;
  // a head's row is requested before the last one's turn is written
  auto row = [&](int h, bool& q) __attribute__((always_inline)) {
    q = h < H;
    return ((q ? b * H + h : b * Hk + (h - H)) * n + t) * 64;
  };
  Half8<DT> nu, nw;
  auto request = [&](int h) __attribute__((always_inline)) {
    if (h >= H + Hk) return;
    bool q;
    const int64_t at = row(h, q);
    const typename DT::T* src = (q ? Q : K) + at;
    nu.load(src + lo);
    nw.load(src + hi);
  };
  request(blockIdx.y);
  for (int h = blockIdx.y; h < H + Hk; h += gridDim.y) {
    float u[8], w[8];
    nu.get(u);
    nw.get(w);
    request(h + gridDim.y);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // interleaved: pair e is (2e, 2e + 1) of the sixteen values u, w; halves: (u[e], w[e])
      float& x = INTERLEAVED ? (e < 4 ? u[2 * e] : w[2 * e - 8]) : u[e];
      float& y = INTERLEAVED ? (e < 4 ? u[2 * e + 1] : w[2 * e - 7]) : w[e];
      const float a = x, c = y;
      x = a * co[e] - c * si[e];
      y = c * co[e] + a * si[e];
    }
    bool q;
    const int64_t at = row(h, q);
    typename DT::T* dst = (q ? Qo : Ko) + at;
    Half8<DT>::store(dst + lo, u);
    Half8<DT>::store(dst + hi, w);
  }
}

}  // namespace

hipError_t launch_rotary(int dtype, int B, int H, int Hk, int n, const void* Q, const void* K, const void* pos,
                         const RotaryPlan& plan, bool interleaved, void* Qo, void* Ko, hipStream_t st) {
  const unsigned tiles = (unsigned)((n + kTok - 1) / kTok);
  const int heads = H + Hk;
  // the sines are formed once per workgroup, so a workgroup takes every head of
  // its tokens unless that leaves compute units idle
  const int64_t wgs = (int64_t)tiles * B;
  int64_t shares = (2048 + wgs - 1) / wgs;
  if (shares > heads) shares = heads;
  const dim3 grid(tiles, (unsigned)shares, (unsigned)B);
  TimedLaunch tl("rotary", st);
#define GA_ROT(DT, I)                                                                                            \
  hipLaunchKernelGGL((k_rotary<DT, I>), grid, dim3(256), 0, st, (const typename DT::T*)Q,                          \
                     (const typename DT::T*)K, pos, plan, H, Hk, n, (typename DT::T*)Qo, (typename DT::T*)Ko)
  if (dtype == 1) {
    if (interleaved) GA_ROT(BF16, true);
    else GA_ROT(BF16, false);
  } else {
    if (interleaved) GA_ROT(F32, true);
    else GA_ROT(F32, false);
  }
#undef GA_ROT
  return hipGetLastError();
}

}  // namespace ga
