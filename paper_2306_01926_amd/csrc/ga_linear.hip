// gfx950 (MI355X) linear attention with a decay for each head.
//
// Per slice (batch b, head h) with the decay l = exp(log_decay[h]) and the
// 64 x 64 state S (key feature by value feature):
//   S_t = l S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t.
// Gradient, from the last token backward:
//   R_t = l R_{t+1} + scale q_t dO_t^T   (R behind the end: the gradient that
//                                         reaches the final state),
//   dK_t = R_t v_t,  dV_t = R_t^T k_t,  dQ_t = scale S_t dO_t,
//   and l R_0 is the gradient of the initial state.
// Each of the three gradients has the forward's form with the roles of the
// tensors changed: dQ walks forward over (dO, V, K) with the state transposed,
// dV and dK walk backward over (K, Q, dO) and (V, dO, Q).
#include <hip/hip_runtime.h>

#include <float.h>
#include <stdint.h>

#include "ga_internal.h"

namespace ga {
namespace {

#include "ga_device.h"

constexpr int kStep = 16;  // tokens staged at a time

// One step's decay of a state value, l x.  Many steps in a row compound what l
// is off by, and 2^-24 of an l near one is large against 1 - l; l - 1 is formed
// without that loss, and l x as x + (l - 1) x with one rounding.  A small l is
// exact enough as it is, and l - 1 would not be.
struct Decay {
  float a, b;  // l = a + b with b 0 or 1
  __device__ __forceinline__ explicit Decay(float log_decay) {
    b = log_decay > -0.5f ? 1.f : 0.f;
    a = b != 0.f ? expm1f(log_decay) : expf(log_decay);
  }
  __device__ __forceinline__ float operator()(float x) const { return fmaf(a, x, b * x); }
};

__device__ __forceinline__ int length_of(const int32_t* lengths, int64_t b, int n) {
  return lengths ? min(max(lengths[b], 0), n) : n;
}

// One wave per slice: lane c holds column c of the state.
struct Walk {
  const void *q, *k, *v;   // roles (see above), [B][H or Hk][n][64]
  bool q_shared, k_shared, v_shared;  // the tensor has Hk heads
  const float *log_decay, *state;
  const int32_t* lengths;
  float* state_out;
  void* out;    // [B][H][n][64] in the storage type, or fp32
  int H, Hk, n;
  float scale;
  bool reverse, transposed, out_f32;
};

template <class DT>
__global__ __launch_bounds__(64) void k_lin_walk(Walk A) {
  using T = typename DT::T;
  __shared__ float qs[kStep][64], ks[kStep][64];
  const int c = threadIdx.x, h = blockIdx.x % A.H;
  const int64_t b = blockIdx.x / A.H, bh = blockIdx.x, bk = b * A.Hk + h / (A.H / A.Hk);
  const int len = length_of(A.lengths, b, A.n);
  const T* q = (const T*)A.q + (A.q_shared ? bk : bh) * A.n * 64;
  const T* k = (const T*)A.k + (A.k_shared ? bk : bh) * A.n * 64;
  const T* v = (const T*)A.v + (A.v_shared ? bk : bh) * A.n * 64;
  const Decay l(A.log_decay[h]);
  float S[64];
#pragma unroll
  for (int a = 0; a < 64; ++a)
    S[a] = !A.state ? 0.f : A.state[bh * 4096 + (A.transposed ? c * 64 + a : a * 64 + c)];
  auto put = [&](int64_t token, float o) {
    const int64_t at = (bh * A.n + token) * 64 + c;
    if (A.out_f32)
      ((float*)A.out)[at] = o;
    else if constexpr (DT::kBits == 16)
      ((T*)A.out)[at] = (T)(pack_bf16x2(o, 0.f) & 0xffffu);
    else
      ((T*)A.out)[at] = o;
  };
  for (int t0 = 0; t0 < len; t0 += kStep) {
    float vr[kStep];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      const int t = min(t0 + u, len - 1);
      const int64_t at = (int64_t)(A.reverse ? len - 1 - t : t) * 64 + c;
      qs[u][c] = DT::load(q, at);
      ks[u][c] = DT::load(k, at);
      vr[u] = DT::load(v, at);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      if (t0 + u >= len) break;
      float o = 0.f;
#pragma unroll
      for (int a = 0; a < 64; ++a) {
        S[a] = A.reverse ? fmaf(ks[u][a] * A.scale, vr[u], S[a]) : fmaf(ks[u][a], vr[u], l(S[a]));
        o = fmaf(qs[u][a], S[a], o);
        if (A.reverse) S[a] = l(S[a]);
      }
      put(A.reverse ? len - 1 - (t0 + u) : t0 + u, A.reverse ? o : o * A.scale);
    }
  }
  for (int t = len; t < A.n; ++t) put(t, 0.f);  // behind the sequence's end
  if (A.state_out) {
#pragma unroll
    for (int a = 0; a < 64; ++a) A.state_out[bh * 4096 + a * 64 + c] = S[a];
  }
}

// One token per sequence: 256 threads per slice, thread (r, g) holds rows
// r + 16 u of the state at columns 4 g .. 4 g + 3.  Bound by the state, 16 KB
// read and 16 KB written per slice; everything is fp32.
template <class DT>
__global__ __launch_bounds__(256) void k_lin_step(const typename DT::T* Q, const typename DT::T* K,
                                                  const typename DT::T* V, const float* log_decay,
                                                  const int32_t* slots, int states, const float* state, int H, int Hk,
                                                  float scale, typename DT::T* O, float* state_out) {
  __shared__ float4 part[4][16];
  const int tid = threadIdx.x, r = tid >> 4, g = tid & 15, h = blockIdx.x % H;
  const int64_t b = blockIdx.x / H, bh = blockIdx.x, bk = b * Hk + h / (H / Hk);
  int64_t slot = b;
  bool live = true;
  if (slots) {
    // a row whose slot lies outside the states, or which an earlier row of the
    // call has taken, is padding
    slot = slots[b];
    bool taken = false;
    for (int64_t i = tid; i < b; i += 256) taken |= slots[i] == slot;
    live = !__syncthreads_or(taken) && slot >= 0 && slot < states;
  }
  if (!live) {
    if (tid < 64) O[bh * 64 + tid] = 0;
    return;
  }
  const int64_t at = (slot * H + h) * 4096 + 4 * g;
  const Decay l(log_decay[h]);
  float4 S[4];
  float q[4], k[4], v[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) S[u] = *(const float4*)(state + at + (r + 16 * u) * 64);
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    q[u] = DT::load(Q, bh * 64 + r + 16 * u);
    k[u] = DT::load(K, bk * 64 + r + 16 * u);
    v[u] = DT::load(V, bk * 64 + 4 * g + u);
  }
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    S[u].x = fmaf(k[u], v[0], l(S[u].x));
    S[u].y = fmaf(k[u], v[1], l(S[u].y));
    S[u].z = fmaf(k[u], v[2], l(S[u].z));
    S[u].w = fmaf(k[u], v[3], l(S[u].w));
    o.x = fmaf(q[u], S[u].x, o.x);
    o.y = fmaf(q[u], S[u].y, o.y);
    o.z = fmaf(q[u], S[u].z, o.z);
    o.w = fmaf(q[u], S[u].w, o.w);
    *(float4*)(state_out + at + (r + 16 * u) * 64) = S[u];
  }
#pragma unroll
  for (int m = 16; m < 64; m <<= 1) {
    o.x += __shfl_xor(o.x, m);
    o.y += __shfl_xor(o.y, m);
    o.z += __shfl_xor(o.z, m);
    o.w += __shfl_xor(o.w, m);
  }
  if ((tid & 63) < 16) part[tid >> 6][g] = o;
  __syncthreads();
  if (tid < 64) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) s += ((const float*)part[w])[tid];
    s *= scale;
    if constexpr (DT::kBits == 16)
      O[bh * 64 + tid] = (uint16_t)(pack_bf16x2(s, 0.f) & 0xffffu);
    else
      O[bh * 64 + tid] = s;
  }
}

// Gradients of shared keys and values: the sum over the query heads of a
// group, in ascending order, rounded once.  Four values per thread.
template <class DT>
__global__ __launch_bounds__(256) void k_lin_heads(const float* __restrict__ part, int H, int Hk, int64_t row4,
                                                   int64_t total4, typename DT::T* __restrict__ out) {
  const int G = H / Hk;
  for (int64_t i = blockIdx.x * 256LL + threadIdx.x; i < total4; i += gridDim.x * 256LL) {
    const int64_t bk = i / row4, x = i - bk * row4;
    const float4* p = (const float4*)part + bk * G * row4 + x;
    float4 s = p[0];
    for (int g = 1; g < G; ++g) {
      const float4 y = p[g * row4];
      s.x += y.x, s.y += y.y, s.z += y.z, s.w += y.w;
    }
    if constexpr (DT::kBits == 16)
      *(u32x2*)(out + 4 * i) = u32x2{pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w)};
    else
      *(float4*)(out + 4 * i) = s;
  }
}

void walk(const LinearDims& d, const Walk& w, hipStream_t st) {
  TimedLaunch tl("lin_walk", st);
  const dim3 grid((unsigned)(d.B * d.H));
  if (d.dtype == 1)
    hipLaunchKernelGGL(k_lin_walk<BF16>, grid, dim3(64), 0, st, w);
  else
    hipLaunchKernelGGL(k_lin_walk<F32>, grid, dim3(64), 0, st, w);
}

}  // namespace

size_t linear_workspace(const LinearDims&) { return 0; }

hipError_t launch_linear(const LinearDims& d, const void* Q, const void* K, const void* V, const float* log_decay,
                         const int32_t* lengths, const float* state, float scale, void* O, float* state_out, void*,
                         hipStream_t st) {
  walk(d, Walk{Q, K, V, false, true, true, log_decay, state, lengths, state_out, O, d.H, d.Hk, d.n, scale, false,
               false, false}, st);
  return hipGetLastError();
}

size_t linear_grad_workspace(const LinearDims& d) {
  return d.H == d.Hk ? 0 : (size_t)d.B * d.H * d.n * 64 * 4;
}

hipError_t launch_linear_grad(const LinearDims& d, const void* Q, const void* K, const void* V, const void* dO,
                              const float* log_decay, const int32_t* lengths, const float* state, const float* dstate,
                              float scale, void* dQ, void* dK, void* dV, float* dstate_out, void* ws, hipStream_t st) {
  const bool grouped = d.H != d.Hk;
  const int64_t row4 = (int64_t)d.n * 16, total4 = (int64_t)d.B * d.Hk * row4;
  const unsigned grid = (unsigned)((total4 + 255) / 256 < 8192 ? (total4 + 255) / 256 : 8192);
  auto heads = [&](void* out) {
    if (!grouped) return;
    TimedLaunch tl("lin_heads", st);
    if (d.dtype == 1)
      hipLaunchKernelGGL(k_lin_heads<BF16>, dim3(grid), dim3(256), 0, st, (const float*)ws, d.H, d.Hk, row4, total4,
                         (uint16_t*)out);
    else
      hipLaunchKernelGGL(k_lin_heads<F32>, dim3(grid), dim3(256), 0, st, (const float*)ws, d.H, d.Hk, row4, total4,
                         (float*)out);
  };
  walk(d, Walk{dO, V, K, false, true, true, log_decay, state, lengths, nullptr, dQ, d.H, d.Hk, d.n, scale, false, true,
               false}, st);
  walk(d, Walk{V, dO, Q, true, false, false, log_decay, dstate, lengths, nullptr, grouped ? ws : dK, d.H, d.Hk, d.n,
               scale, true, true, grouped}, st);
  heads(dK);
  walk(d, Walk{K, Q, dO, true, false, false, log_decay, dstate, lengths, dstate_out, grouped ? ws : dV, d.H, d.Hk, d.n,
               scale, true, false, grouped}, st);
  heads(dV);
  return hipGetLastError();
}

hipError_t launch_linear_step(const LinearDims& d, const void* Q, const void* K, const void* V, const float* log_decay,
                              const int32_t* slots, int states, const float* state, float scale, void* O,
                              float* state_out, hipStream_t st) {
  TimedLaunch tl("lin_step", st);
  const dim3 grid((unsigned)(d.B * d.H));
  if (d.dtype == 1)
    hipLaunchKernelGGL(k_lin_step<BF16>, grid, dim3(256), 0, st, (const uint16_t*)Q, (const uint16_t*)K,
                       (const uint16_t*)V, log_decay, slots, states, state, d.H, d.Hk, scale, (uint16_t*)O, state_out);
  else
    hipLaunchKernelGGL(k_lin_step<F32>, grid, dim3(256), 0, st, (const float*)Q, (const float*)K, (const float*)V,
                       log_decay, slots, states, state, d.H, d.Hk, scale, (float*)O, state_out);
  return hipGetLastError();
}

}  // namespace ga
