// gfx950 (MI355X) norms around a block, fused with its gate and the residual's
// scale, and their gradient.
//
// For every token (row of W features), x the residual stream, f the block's
// output:
//   u = post-norm of f (f itself without one),
//   y = a x + b g * u          (a, b scalars, g a gate per feature),
//   h = pre-norm of y          (the next block's input),
//   norm(z) = w * (z - mean z) / sqrt(var z + eps) + c     (layer)
//           = w * z / sqrt(mean z^2 + eps) + c             (rms).
// Gradient, with zn the normalised row, r its 1 / sqrt(...) and P the
// projection P(d) = r (d - zn mean(d zn) [- mean d for layer]):
//   D  = dy + P_y(w_pre dh),   dx = a D,
//   df = P_f(w_post b g D),    dw_post = sum b g D fn,  dc_post = sum b g D,
//   dg = sum b u D,            dw_pre  = sum dh yn,     dc_pre  = sum dh.
// The gradient forms y and both norms again from x and f (the same bytes as
// reading a stored y), so nothing is kept from the forward pass.
//
// Both are bound by HBM: 4 rows of W values moved per token forward (x, f in,
// y, h out), 6 backward (D = 512, 128000 tokens, bf16: 112 us, 4.7 TB/s; gradient
// 166 us, 4.7 TB/s; a copy runs at 5.3).  A row lives in the registers of TPR threads, eight
// consecutive features each, so it is read once; the variance is the mean
// square about the mean, formed from those registers (two sums), all in fp32.
// One wave holds a row of up to 512 features and reduces by lane exchanges
// only.  Parameter gradients are summed over a workgroup's rows in registers,
// its teams are added in LDS, and a second launch adds the workgroups' rows in
// ascending order: no atomics, the same bits on every run.
#include <hip/hip_runtime.h>

#include <float.h>
#include <stdint.h>

#include "ga_internal.h"

namespace ga {
namespace {

#include "ga_device.h"

constexpr int kE = 8;  // features per thread

// Eight features of one row from column c (beyond W: zeros), as they come from
// memory: requested a row ahead, converted where they are used.  VEC: W is a
// multiple of eight, so every group of eight is whole and 16-byte aligned.  Else
// groups are read and written in one piece at any alignment (global memory
// allows it); a row's last, incomplete one is read with the features before it
// and shifted where it is used (rows of fewer than eight: by single features),
// and written by single features.
struct __attribute__((packed, aligned(2))) Piece {
  u32x4 w;
};
template <class DT, bool VEC>
struct Eight {
  using T = typename DT::T;
  static constexpr int kWords = DT::kBits == 16 ? 1 : 2, kPer = kE / kWords;  // 16-byte words, features in one
  uint32_t w[4 * kWords];
  int behind;  // features read that lie before column c; kE: none is wanted

  __device__ __forceinline__ void load(const T* p, int c, int W) {
    if (VEC) {
      if (c < W) {
        put(p + c);
      } else {
        zero();
      }
      return;
    }
    behind = min(max(c - (W - kE), 0), kE);
    if (W >= kE) {
      put(p + min(c, W - kE));
    } else {
      zero();
      behind = 0;
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        if (c + e >= W) continue;
        if constexpr (DT::kBits == 16)
          w[e / 2] |= (uint32_t)p[c + e] << (16 * (e & 1));
        else
          w[e] = __float_as_uint(p[c + e]);
      }
    }
  }
  // shifts the group into place, before get: few lanes need it, and a wave with
  // none of them jumps over it
  __device__ __forceinline__ void settle() {
    if constexpr (!VEC) {
      constexpr int kN = 4 * kWords;
      if (!__any(behind != 0)) return;
#pragma unroll
      for (int s = kE; s >= 1; s /= 2) {  // by 8, 4, 2 and 1 features
        const bool on = (behind & s) != 0;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          uint32_t y;
          if constexpr (DT::kBits == 16) {
            const uint32_t hi = i + 1 < kN ? w[i + 1 < kN ? i + 1 : 0] : 0u;
            y = s == 1 ? w[i] >> 16 | hi << 16 : (i + s / 2 < kN ? w[i + s / 2 < kN ? i + s / 2 : 0] : 0u);
          } else {
            y = i + s < kN ? w[i + s < kN ? i + s : 0] : 0u;
          }
          w[i] = on ? y : w[i];
        }
      }
    }
  }
  __device__ __forceinline__ void get(float (&v)[kE]) const {
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      if constexpr (DT::kBits == 16)
        v[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
      else
        v[e] = __uint_as_float(w[e]);
    }
  }

 private:
  __device__ __forceinline__ void put(const T* p) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const u32x4 y = VEC ? *(const u32x4*)(p + kPer * i) : ((const Piece*)(p + kPer * i))->w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * i + j] = y[j];
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < 4 * kWords; ++i) w[i] = 0u;
  }
};
template <class DT, bool VEC>
__device__ __forceinline__ void load8(const typename DT::T* p, int c, int W, float (&v)[kE]) {
  Eight<DT, VEC> x;
  x.load(p, c, W);
  x.settle();
  x.get(v);
}

// The outputs are rounded once, to nearest even (bf16), here.
template <class DT, bool VEC>
__device__ __forceinline__ void store8(typename DT::T* p, int c, int W, const float (&v)[kE]) {
  using E = Eight<DT, VEC>;
  u32x4 w[E::kWords];
#pragma unroll
  for (int e = 0; e < kE; e += 2) {
    if constexpr (DT::kBits == 16) {
      w[0][e / 2] = pack_bf16x2(v[e], v[e + 1]);
    } else {
      w[e / 4][e % 4] = __float_as_uint(v[e]);
      w[e / 4][e % 4 + 1] = __float_as_uint(v[e + 1]);
    }
  }
  if (VEC ? c < W : c + kE <= W) {
#pragma unroll
    for (int i = 0; i < E::kWords; ++i) {
      if (VEC)
        *(u32x4*)(p + c + E::kPer * i) = w[i];
      else
        ((Piece*)(p + c + E::kPer * i))->w = w[i];
    }
  } else if (!VEC) {
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      if (c + e >= W) continue;
      if constexpr (DT::kBits == 16)
        p[c + e] = (uint16_t)(w[0][e / 2] >> (16 * (e & 1)));
      else
        p[c + e] = v[e];
    }
  }
}

// The sum over groups of min(TPR, 64) lanes, in each of them, by lane exchanges
// of the VALU (an exchange through LDS takes ten times as long, and a row waits
// for up to eight sums one after another).
template <int TPR>
__device__ __forceinline__ float lanes_sum(float x) {
  x += __int_as_float(dpp<kXor1>(__float_as_int(x)));
  x += __int_as_float(dpp<kXor2>(__float_as_int(x)));
  x += __int_as_float(dpp<kHalfMirror>(__float_as_int(x)));
  if constexpr (TPR >= 16) x += __int_as_float(dpp<kMirror>(__float_as_int(x)));
  if constexpr (TPR >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  if constexpr (TPR >= 64) {
    const u32x2 q = halves(__float_as_uint(x));
    x = __uint_as_float(q[0]) + __uint_as_float(q[1]);
  }
  return x;
}

// Sums of two values over the TPR threads of a team, in every thread of it.
// Teams of more than a wave exchange through red[16], one entry per wave.
// The calls inside one row's work have a red each, and rows alternate between
// two sets of them: whoever writes an entry again has passed the barrier of a
// later call (in the next row at the latest), before which every wave had read
// it.
template <int TPR>
__device__ __forceinline__ float2 team_sum(float a, float b, float2* red) {
  a = lanes_sum<TPR>(a);
  b = lanes_sum<TPR>(b);
  if constexpr (TPR > 64) {
    constexpr int kW = TPR / 64;  // waves per team
    const int wave = threadIdx.x >> 6, first = wave / kW * kW;
    if ((threadIdx.x & 63) == 0) red[wave] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < kW; ++w) {
      const float2 r = red[first + w];
      a += r.x;
      b += r.y;
    }
  }
  return make_float2(a, b);
}

constexpr int wg_threads(int TPR) { return TPR < 256 ? 256 : TPR; }

// z -> zn = (z - mean) r in place; returns r.  red: a buffer of this call's own.
template <int TPR>
__device__ __forceinline__ float normalise(float (&z)[kE], int c, int W, float invW, bool layer, float eps,
                                           float2 (*red)[16]) {
  if (layer) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < kE; ++e) s += z[e];
    const float mean = team_sum<TPR>(s, 0.f, red[0]).x * invW;
#pragma unroll
    for (int e = 0; e < kE; ++e) z[e] = c + e < W ? z[e] - mean : 0.f;
  }
  float q = 0.f;
#pragma unroll
  for (int e = 0; e < kE; ++e) q = fmaf(z[e], z[e], q);
  const float r = rsqrtf(team_sum<TPR>(q, 0.f, red[1]).x * invW + eps);
#pragma unroll
  for (int e = 0; e < kE; ++e) z[e] *= r;
  return r;
}

// d -> P(d) in place (see the head of the file): mz = mean(d zn), md = mean d or 0.
__device__ __forceinline__ void project(float (&d)[kE], const float (&zn)[kE], float r, float mz, float md, int c, int W) {
#pragma unroll
  for (int e = 0; e < kE; ++e) d[e] = c + e < W ? r * (d[e] - fmaf(zn[e], mz, md)) : 0.f;
}

template <class DT>
struct NormArgs {
  using T = typename DT::T;
  const T *X, *F, *post_w, *post_b, *gate, *pre_w, *pre_b;
  int64_t rows;      // tokens
  int n, W;          // tokens per batch, features
  int gate_batches;  // 0: no gate, 1: one for all tokens, B: one per batch
  float invW, eps, a, b;
  bool layer;
};

template <class DT, int TPR, bool VEC>
__global__ __launch_bounds__(wg_threads(TPR)) void k_norm(NormArgs<DT> A, typename DT::T* __restrict__ Y,
                                                          typename DT::T* __restrict__ Ho) {
  __shared__ float2 reds[2][4][16];
  constexpr int kTeams = wg_threads(TPR) / TPR;
  const int team = threadIdx.x / TPR, c = (threadIdx.x % TPR) * kE, W = A.W;
  float pw[kE], pb[kE], gt[kE], qw[kE], qb[kE];
  if (A.post_w) load8<DT, VEC>(A.post_w, c, W, pw);
  if (A.post_b) load8<DT, VEC>(A.post_b, c, W, pb);
  if (A.gate_batches == 1) load8<DT, VEC>(A.gate, c, W, gt);
  if (Ho) load8<DT, VEC>(A.pre_w, c, W, qw);
  if (Ho && A.pre_b) load8<DT, VEC>(A.pre_b, c, W, qb);
  int parity = 0;
  const int64_t step = (int64_t)gridDim.x * kTeams;
  Eight<DT, VEC> nx, nf, ng;  // the next row
  auto request = [&](int64_t row0) __attribute__((always_inline)) {
    const int64_t row = min(row0 + team, A.rows - 1);
    nx.load(A.X + row * W, c, W);
    if (A.F) nf.load(A.F + row * W, c, W);
    if (A.gate_batches > 1)
      ng.load(A.gate + (A.rows <= INT32_MAX ? (int64_t)((uint32_t)row / (uint32_t)A.n) : row / A.n) * W, c, W);
  };
  request((int64_t)blockIdx.x * kTeams);
  // every team makes the same number of turns (barriers inside)
  for (int64_t row0 = (int64_t)blockIdx.x * kTeams; row0 < A.rows; row0 += step) {
    float2(*red)[16] = reds[parity];
    parity ^= 1;
    const bool live = row0 + team < A.rows;
    const int64_t row = min(row0 + team, A.rows - 1);
    float y[kE], u[kE];
    nx.settle(), nx.get(y);
    if (A.F) nf.settle(), nf.get(u);
    if (A.gate_batches > 1) ng.settle(), ng.get(gt);
    request(row0 + step);
#pragma unroll
    for (int e = 0; e < kE; ++e) y[e] *= A.a;
    if (A.F) {
      if (A.post_w) {
        normalise<TPR>(u, c, W, A.invW, A.layer, A.eps, red);
#pragma unroll
        for (int e = 0; e < kE; ++e) u[e] = fmaf(u[e], pw[e], A.post_b ? pb[e] : 0.f);
      }
#pragma unroll
      for (int e = 0; e < kE; ++e) y[e] = fmaf(A.gate_batches ? A.b * gt[e] : A.b, u[e], y[e]);
    }
    if (Y && live) store8<DT, VEC>(Y + row * W, c, W, y);
    if (Ho) {
      normalise<TPR>(y, c, W, A.invW, A.layer, A.eps, red + 2);
#pragma unroll
      for (int e = 0; e < kE; ++e) y[e] = fmaf(y[e], qw[e], A.pre_b ? qb[e] : 0.f);
      if (live) store8<DT, VEC>(Ho + row * W, c, W, y);
    }
  }
}

// Rows of one batch group are spread over `split` workgroups, or a workgroup
// takes `each` whole groups (split == 1).  part: [gridDim.x][4][W] sums of
// dpost_w, dpost_b, dpre_w, dpre_b; gpart: [groups][split][W] sums of dgate.
struct NormParts {
  float *part, *gpart;
  int groups, split, each;
  int64_t group_rows;
};

// A thread's sums of one parameter's gradient over the rows, in registers or in
// LDS.
template <bool LDS>
struct Sums {
  float v[LDS ? 1 : kE];
  float* at;
  __device__ __forceinline__ void start(float* lds) {
    at = lds + threadIdx.x;
#pragma unroll
    for (int e = 0; e < kE; ++e) (LDS ? at[1024 * e] : v[LDS ? 0 : e]) = 0.f;
  }
  __device__ __forceinline__ void add(int e, float a, float b) {
    float& s = LDS ? at[1024 * e] : v[LDS ? 0 : e];
    s = fmaf(a, b, s);
  }
  __device__ __forceinline__ void get(float (&x)[kE]) const {
#pragma unroll
    for (int e = 0; e < kE; ++e) x[e] = LDS ? at[1024 * e] : v[LDS ? 0 : e];
  }
};

template <int TPR>
__device__ __forceinline__ void team_store(const float (&v)[kE], float* buf, float* dst, int W) {
  constexpr int kT = wg_threads(TPR), kTeams = kT / TPR;
  if (kTeams == 1) {
    store8<F32, false>(dst, threadIdx.x * kE, W, v);
    return;
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kE; ++e) buf[(threadIdx.x / TPR) * (TPR * kE) + (threadIdx.x % TPR) * kE + e] = v[e];
  __syncthreads();
  for (int col = threadIdx.x; col < W; col += kT) {
    float s = 0.f;
#pragma unroll
    for (int t = 0; t < kTeams; ++t) s += buf[t * (TPR * kE) + col];
    dst[col] = s;
  }
}

// BIAS: the gradients of the norms' biases are asked for.
// Threads of a team of 1024 have 128 registers each: they keep the sums in LDS,
// read the parameters again (from the caches) where they use them and the rows
// where they begin them (D = 8192, 4000 rows, bf16: 123 us, and 279 with all of
// it in registers, most of them spilled).
template <class DT, int TPR, bool VEC, bool BIAS>
__global__ __launch_bounds__(wg_threads(TPR)) void k_norm_grad(NormArgs<DT> A, const typename DT::T* __restrict__ dY,
                                                               const typename DT::T* __restrict__ dH,
                                                               typename DT::T* __restrict__ dX,
                                                               typename DT::T* __restrict__ dF, NormParts P) {
  constexpr int kT = wg_threads(TPR), kTeams = kT / TPR;
  using Raw = Eight<DT, VEC>;
  __shared__ float2 reds[2][6][16];
  __shared__ float buf[kTeams > 1 ? kT * kE : 1];
  const int team = threadIdx.x / TPR, c = (threadIdx.x % TPR) * kE, W = A.W;
  constexpr bool kLds = TPR == 1024;
  Raw pw, pb, gt, qw;  // (as stored: half the registers)
  auto fetch = [&](Raw& r, const typename DT::T* p) __attribute__((always_inline)) { r.load(p, c, W), r.settle(); };
  auto param = [&](Raw& r, const typename DT::T* p, float(&v)[kE]) __attribute__((always_inline)) {
    if (kLds) fetch(r, p);
    r.get(v);
  };
  if (!kLds && A.post_w) fetch(pw, A.post_w);
  if (!kLds && A.post_b) fetch(pb, A.post_b);
  if (!kLds && dH) fetch(qw, A.pre_w);
  constexpr int kSums = kLds ? kT * kE : 0;
  __shared__ float lds[kLds ? 4 * kSums : 1];
  Sums<kLds> spw, sqw, spb, sqb;
  spw.start(lds), sqw.start(lds + kSums);
  if (BIAS) spb.start(lds + 2 * kSums), sqb.start(lds + 3 * kSums);
  float sg[kE];

  int parity = 0;
  for (int i = 0; i < P.each; ++i) {
    const int grp = P.split > 1 ? blockIdx.x / P.split : blockIdx.x * P.each + i;
    if (grp >= P.groups) break;  // the same for every thread
    const int share = P.split > 1 ? blockIdx.x % P.split : 0;
#pragma unroll
    for (int e = 0; e < kE; ++e) sg[e] = 0.f;
    const typename DT::T* gate = A.gate_batches ? A.gate + (A.gate_batches > 1 ? (int64_t)grp * W : 0) : nullptr;
    if (!kLds && gate) fetch(gt, gate);
    Raw nx, nf, ny, nh;  // the next row
    auto request = [&](int64_t r0) __attribute__((always_inline)) {
      const int64_t at = (grp * P.group_rows + min(r0 + team, P.group_rows - 1)) * W;
      nx.load(A.X + at, c, W);
      if (A.F) nf.load(A.F + at, c, W);
      if (dY) ny.load(dY + at, c, W);
      if (dH) nh.load(dH + at, c, W);
    };
    if (!kLds) request((int64_t)share * kTeams);
    for (int64_t r0 = (int64_t)share * kTeams; r0 < P.group_rows; r0 += (int64_t)P.split * kTeams) {
      float2(*red)[16] = reds[parity];
      parity ^= 1;
      // a team behind the last row works on it again, and its sums count nothing
      const float live = r0 + team < P.group_rows ? 1.f : 0.f;
      const int64_t row = grp * P.group_rows + min(r0 + team, P.group_rows - 1);
      if (kLds) request(r0);
      float y[kE], fn[kE], d[kE], dh[kE], w[kE], g[kE], rf = 0.f;
      nx.settle(), nx.get(y);
      if (A.F) nf.settle(), nf.get(fn);
      if (dY) {
        ny.settle(), ny.get(d);
      } else {
#pragma unroll
        for (int e = 0; e < kE; ++e) d[e] = 0.f;
      }
      if (dH) nh.settle(), nh.get(dh);
      if (!kLds) request(r0 + (int64_t)P.split * kTeams);
#pragma unroll
      for (int e = 0; e < kE; ++e) y[e] *= A.a;
      // u = w fn + c, formed where it is used
      auto branch = [&](float(&u)[kE]) __attribute__((always_inline)) {
        if (A.post_w) {
          param(pw, A.post_w, u);
          float s[kE];
          if (A.post_b) param(pb, A.post_b, s);
#pragma unroll
          for (int e = 0; e < kE; ++e) u[e] = fmaf(fn[e], u[e], A.post_b ? s[e] : 0.f);
        } else {
#pragma unroll
          for (int e = 0; e < kE; ++e) u[e] = fn[e];
        }
      };
      auto gates = [&]() __attribute__((always_inline)) {
        if (gate) param(gt, gate, g);
#pragma unroll
        for (int e = 0; e < kE; ++e) g[e] = gate ? A.b * g[e] : A.b;
      };
      if (A.F) {
        if (A.post_w) rf = normalise<TPR>(fn, c, W, A.invW, A.layer, A.eps, red);
        branch(w);
        gates();
#pragma unroll
        for (int e = 0; e < kE; ++e) y[e] = fmaf(g[e], w[e], y[e]);
      }
      if (dH) {
        // the sums that the projection needs go with those of the norm
        float sd = 0.f;
        param(qw, A.pre_w, w);
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          w[e] *= dh[e];  // (zeros beyond W)
          sd += w[e];
        }
        float md = 0.f;
        if (A.layer) {
          float s = 0.f;
#pragma unroll
          for (int e = 0; e < kE; ++e) s += y[e];
          const float2 m = team_sum<TPR>(s, sd, red[2]);
          md = m.y * A.invW;
#pragma unroll
          for (int e = 0; e < kE; ++e) y[e] = c + e < W ? y[e] - m.x * A.invW : 0.f;
        }
        float q = 0.f, s = 0.f;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          q = fmaf(y[e], y[e], q);
          s = fmaf(w[e], y[e], s);
        }
        const float2 m = team_sum<TPR>(q, s, red[3]);
        const float rh = rsqrtf(m.x * A.invW + A.eps);
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          y[e] *= rh;
          dh[e] *= live;
          sqw.add(e, dh[e], y[e]);
          if (BIAS) sqb.add(e, 1.f, dh[e]);
        }
        project(w, y, rh, rh * m.y * A.invW, md, c, W);
#pragma unroll
        for (int e = 0; e < kE; ++e) d[e] += w[e];
      }
      if (A.F) {
        float du[kE];
        branch(w);
        gates();
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          sg[e] = fmaf(live * A.b * d[e], w[e], sg[e]);
          du[e] = g[e] * d[e];
        }
        if (A.post_w) {
          param(pw, A.post_w, w);
          float s = 0.f, sd = 0.f;
#pragma unroll
          for (int e = 0; e < kE; ++e) {
            spw.add(e, live * du[e], fn[e]);
            if (BIAS) spb.add(e, live, du[e]);
            du[e] = c + e < W ? du[e] * w[e] : 0.f;
            s = fmaf(du[e], fn[e], s);
            sd += du[e];
          }
          const float2 m = team_sum<TPR>(s, sd, red[5]);
          project(du, fn, rf, m.x * A.invW, A.layer ? m.y * A.invW : 0.f, c, W);
        }
        if (dF && live != 0.f) store8<DT, VEC>(dF + row * W, c, W, du);
      }
      if (dX && live != 0.f) {
#pragma unroll
        for (int e = 0; e < kE; ++e) d[e] *= A.a;
        store8<DT, VEC>(dX + row * W, c, W, d);
      }
    }
    if (P.gpart) team_store<TPR>(sg, buf, P.gpart + ((int64_t)grp * P.split + share) * W, W);
  }
  if (P.part) {
    float* dst = P.part + (int64_t)blockIdx.x * 4 * W;
    auto store = [&](const Sums<kLds>& s, int which) __attribute__((always_inline)) {
      float v[kE];
      s.get(v);
      team_store<TPR>(v, buf, dst + (int64_t)which * W, W);
    };
    if (A.post_w) {
      store(spw, 0);
      if (BIAS) store(spb, 1);
    }
    if (dH) {
      store(sqw, 2);
      if (BIAS) store(sqb, 3);
    }
  }
}

// out[col] = sum over parts p of src[p stride + col] for the four parameters'
// sums (of all workgroups) and each group's gate (of its workgroups): in
// ascending order within each of the interleaved shares that a column's threads
// take, 32 columns and up to 32 shares to a workgroup.  grid: ceil(W / 32)
// blocks of columns, times 4 parameters and the groups.
struct NormOuts {
  float* out[5];
};
__global__ __launch_bounds__(1024) void k_norm_params(const float* __restrict__ part, const float* __restrict__ gpart,
                                                      int wgs, int split, int W, NormOuts O) {
  __shared__ float buf[32][33];
  const int blocks = (W + 31) / 32, row = (int)(blockIdx.x / blocks), which = min(row, 4);
  if (!O.out[which]) return;
  const int64_t group = row - which;
  float* out = O.out[which] + group * W;
  const float* src = which == 4 ? gpart + group * split * W : part + (int64_t)which * W;
  const int64_t stride = which == 4 ? W : 4 * (int64_t)W;
  const int count = which == 4 ? split : wgs, shares = blockDim.x >> 5;
  const int cl = threadIdx.x & 31, s = threadIdx.x >> 5, col = (int)(blockIdx.x - (unsigned)row * blocks) * 32 + cl;
  float v = 0.f;
  if (col < W) {
#pragma unroll 8
    for (int p = s; p < count; p += shares) v += src[p * stride + col];
  }
  buf[s][cl] = v;
  __syncthreads();
  if (s == 0 && col < W) {
    float t = 0.f;
    for (int k = 0; k < shares; ++k) t += buf[k][cl];
    out[col] = t;
  }
}

int threads_per_row(int W) {
  int t = 8;
  while (t * kE < W) t *= 2;
  return t;
}

// The gradient's grouping of rows into workgroups: as many as are resident at
// once (the registers hold two waves per SIMD), since each writes a row of
// parameter sums (D = 4096: 102 us with 256 workgroups of 512 threads, 112 with
// 512; D = 1024: 81 us with 512 of 256, 109 with 256).  A gate per batch keeps a
// workgroup inside one batch, or gives it several whole ones where batches are
// many.
int norm_wgs(int tpr) { return tpr > 256 ? 256 : 512; }
NormParts parts_of(const NormDims& d) {
  NormParts p{};
  p.groups = d.gate_batches > 1 ? d.gate_batches : 1;
  p.group_rows = d.gate_batches > 1 ? d.n : (int64_t)d.B * d.n;
  const int tpr = threads_per_row(d.W), teams = wg_threads(tpr) / tpr;
  const int64_t most = (p.group_rows + teams - 1) / teams;
  int64_t split = norm_wgs(tpr) / p.groups;
  p.split = (int)(split < 1 ? 1 : (split > most ? most : split));
  p.each = p.split > 1 ? 1 : (p.groups + norm_wgs(tpr) - 1) / norm_wgs(tpr);
  return p;
}
int wgs_of(const NormParts& p) { return p.split > 1 ? p.groups * p.split : (p.groups + p.each - 1) / p.each; }

template <class DT>
NormArgs<DT> args_of(const NormDims& d, const NormTensors& t) {
  using T = typename DT::T;
  return NormArgs<DT>{(const T*)t.X,    (const T*)t.F,     (const T*)t.post_w, (const T*)t.post_b, (const T*)t.gate,
                      (const T*)t.pre_w, (const T*)t.pre_b, (int64_t)d.B * d.n, d.n,                d.W,
                      d.gate_batches,   1.0f / (float)d.W, d.eps,              d.a,                d.b,
                      d.layer != 0};
}

#define GA_NORM_TPR(DT, VEC, CALL) \
  switch (threads_per_row(d.W)) {  \
    case 8: CALL(DT, 8, VEC); break;     \
    case 16: CALL(DT, 16, VEC); break;   \
    case 32: CALL(DT, 32, VEC); break;   \
    case 64: CALL(DT, 64, VEC); break;   \
    case 128: CALL(DT, 128, VEC); break; \
    case 256: CALL(DT, 256, VEC); break; \
    case 512: CALL(DT, 512, VEC); break; \
    default: CALL(DT, 1024, VEC); break; \
  }
#define GA_NORM_ALL(CALL)                        \
  if (d.dtype == 1 && d.W % kE == 0) {           \
    GA_NORM_TPR(BF16, true, CALL)                \
  } else if (d.dtype == 1) {                     \
    GA_NORM_TPR(BF16, false, CALL)               \
  } else if (d.W % kE == 0) {                    \
    GA_NORM_TPR(F32, true, CALL)                 \
  } else {                                       \
    GA_NORM_TPR(F32, false, CALL)                \
  }

}  // namespace

int norm_max_width() { return 1024 * kE; }

hipError_t launch_norm(const NormDims& d, const NormTensors& t, void* Y, void* H, hipStream_t st) {
  const int tpr = threads_per_row(d.W), teams = wg_threads(tpr) / tpr;
  const int64_t rows = (int64_t)d.B * d.n, wgs = (rows + teams - 1) / teams;
  const unsigned grid = (unsigned)(wgs < 4096 ? wgs : 4096);
  TimedLaunch tl("norm", st);
#define GA_CALL(DT, TPR, VEC)                                                                               \
  hipLaunchKernelGGL((k_norm<DT, TPR, VEC>), dim3(grid), dim3(wg_threads(TPR)), 0, st, args_of<DT>(d, t),    \
                     (typename DT::T*)Y, (typename DT::T*)H)
  GA_NORM_ALL(GA_CALL)
#undef GA_CALL
  return hipGetLastError();
}

size_t norm_grad_workspace(const NormDims& d) {
  const NormParts p = parts_of(d);
  return ((size_t)wgs_of(p) * 4 + (size_t)p.groups * p.split) * d.W * 4;
}

hipError_t launch_norm_grad(const NormDims& d, const NormTensors& t, const void* dY, const void* dH, void* dX,
                            void* dF, float* const out[5], void* ws, hipStream_t st) {
  NormParts p = parts_of(d);
  const int wgs = wgs_of(p);
  const bool params = out[0] || out[1] || out[2] || out[3];
  p.part = params ? (float*)ws : nullptr;
  // a group of one share is the result itself
  p.gpart = !out[4] ? nullptr : (p.split == 1 ? out[4] : (float*)ws + (size_t)wgs * 4 * d.W);
  {
    TimedLaunch tl("norm_grad", st);
#define GA_CALL(DT, TPR, VEC)                                                                                     \
  do {                                                                                                             \
    if (out[1] || out[3])                                                                                          \
      hipLaunchKernelGGL((k_norm_grad<DT, TPR, VEC, true>), dim3((unsigned)wgs), dim3(wg_threads(TPR)), 0, st,      \
                         args_of<DT>(d, t), (const typename DT::T*)dY, (const typename DT::T*)dH,                  \
                         (typename DT::T*)dX, (typename DT::T*)dF, p);                                             \
    else                                                                                                           \
      hipLaunchKernelGGL((k_norm_grad<DT, TPR, VEC, false>), dim3((unsigned)wgs), dim3(wg_threads(TPR)), 0, st,     \
                         args_of<DT>(d, t), (const typename DT::T*)dY, (const typename DT::T*)dH,                  \
                         (typename DT::T*)dX, (typename DT::T*)dF, p);                                             \
  } while (0)
    GA_NORM_ALL(GA_CALL)
#undef GA_CALL
  }
  const bool gate = out[4] && p.split > 1;
  if (params || gate) {
    TimedLaunch tl("norm_params", st);
    NormOuts o{{out[0], out[1], out[2], out[3], gate ? out[4] : nullptr}};
    // eight parts to a share, which are requested at once
    unsigned shares = 2;
    while (shares < 32 && shares * 8 < (unsigned)wgs) shares *= 2;
    hipLaunchKernelGGL(k_norm_params, dim3((unsigned)((d.W + 31) / 32 * (gate ? 4 + p.groups : 4))), dim3(32 * shares), 0,
                       st, p.part, p.gpart, wgs, p.split, d.W, o);
  }
  return hipGetLastError();
}

}  // namespace ga
