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

// ---------------------------------------------------------------- bf16, by chunks
//
// A chunk of 64 tokens is computed from the state before it:
//   O = scale ((Q K^T * D) V + diag(l^{i+1}) Q S),  D_ij = l^{i-j} for j <= i,
//   S' = l^64 S + sum_j l^{63-j} k_j v_j^T,
// all four products on the matrix cores.  A workgroup of four waves walks the
// chunks of one slice, or of one of P segments of it; wave (rb, ch) owns the
// 32 tokens rb and the 32 value features ch of the output, and the quadrant
// (features 32 rb of k) x (features 32 ch of v) of the state in 16 registers.
//
// Products are formed transposed (K Q^T, V^T P^T, ...), so the scores' result
// registers are the next product's operand as they are: no LDS round trip.
// The value rows feeding the last product are permuted so that a lane ends with
// 16 consecutive features of one token (32 bytes, stored from registers).
// K and V rows sit in LDS as they come (16-byte granules XOR-swizzled by row);
// the operands that need a column of them come from transposing LDS reads.
//
// Roundings: the scores after decay and the state that Q meets are rounded to
// bf16, as the matrix cores need (each term of an output passes one of the
// two); the state itself is fp32, and the decayed keys that it sums are kept
// as two bf16 parts (16 significant bits), two products each.
constexpr int kC = 64;         // tokens per chunk
constexpr int kTile = kC * 128;  // bytes of a chunk's rows of 64 bf16
constexpr float kLog2e = 1.4426950408889634f;

// l^x as 2^(g x), g = log2 l, bounded so that l = 0 (log_decay = -inf) gives
// l^0 = 1 and l^x = 0 without a product of zero and infinity.
__device__ __forceinline__ float decay_log2(float log_decay) { return fmaxf(log_decay * kLog2e, -1.0e30f); }
__device__ __forceinline__ float decay_pow(float g, float x) { return __builtin_amdgcn_exp2f(g * x); }

typedef short i16x4 __attribute__((ext_vector_type(4)));
// Transposing LDS read (ds_read_b64_tr_b16): within 16 lanes, lane i receives
// element i % 4 of the 8-byte rows addressed by lanes 4 j + i / 4, j = 0..3.
__device__ __forceinline__ u32x2 lds_tr16(const unsigned char* p) {
  const i16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p);
  return __builtin_bit_cast(u32x2, v);
}
__device__ __forceinline__ u32x4 join(u32x2 a, u32x2 b) { return u32x4{a[0], a[1], b[0], b[1]}; }
__device__ __forceinline__ f32x16 mfma(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                 0, 0);
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int v = 0; v < 16; ++v) z[v] = 0.f;
  return z;
}

// Byte offset of 16-byte granule q of row r of a tile: the key takes all eight
// values on eight consecutive rows, so that reads of one granule of many rows
// and transposing reads of four rows spread over the banks.
__device__ __forceinline__ int tkey(int r) { return (r & 7) ^ ((r >> 3) & 1); }
__device__ __forceinline__ int toff(int r, int q) { return r * 128 + ((q ^ tkey(r)) << 4); }

struct Chunked {
  const uint16_t *q, *k, *v;          // roles (see the head of the file)
  bool q_shared, k_shared, v_shared;  // the tensor has Hk heads
  const float *log_decay, *state;
  const int32_t* lengths;
  float* seg;        // [B H][P][64][64]: local states (STATES), then the states before each segment; P > 1 only
  float* state_out;
  void* out;
  int H, Hk, n, P, cps;  // segments per slice, chunks per segment
  float scale;
  bool transposed, out_f32;
};

// REV walks from a sequence's last token to its first; its state is R of the
// head of the file times l, the carry to the token before: a token's own decay
// is behind it, so the exponents are one lower at the output and one higher in
// the sum, and the scale sits in the sum.
// STATES: the local states of the segments alone (from zero; no output).
template <bool REV, bool STATES>
__global__ __launch_bounds__(256, 2) void k_lin_chunk(Chunked A) {
  constexpr int kTiles = STATES ? 3 : 4;  // V, K hi, K lo (decayed), K
  __shared__ __attribute__((aligned(16))) unsigned char lds[2 * kTiles * kTile + (STATES ? 0 : 2 * kTile)];
  const int nseg = STATES ? A.P - 1 : A.P;
  const int64_t bh = blockIdx.x / nseg;
  const int p = (int)(blockIdx.x - bh * nseg);
  const int h = (int)(bh % A.H);
  const int64_t b = bh / A.H, bk = b * A.Hk + h / (A.H / A.Hk);
  const int len = length_of(A.lengths, b, A.n);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int rb = wave & 1, ch = wave >> 1, r = lane & 31, hf = lane >> 5;
  const uint16_t* q = A.q + (A.q_shared ? bk : bh) * A.n * 64;
  const uint16_t* k = A.k + (A.k_shared ? bk : bh) * A.n * 64;
  const uint16_t* v = A.v + (A.v_shared ? bk : bh) * A.n * 64;
  const float g = decay_log2(A.log_decay[h]);
  const int c0 = p * A.cps, c1 = min(c0 + A.cps, (len + kC - 1) / kC);
  auto row = [&](int t) __attribute__((always_inline)) {  // first feature of walk position t (clamped)
    const int x = min(t, len - 1);
    return (int64_t)(REV ? len - 1 - x : x) * 64;
  };

  // the state's quadrant: S[a][c], a = 32 rb + r, c = 32 ch + 16 hf + 0..15
  const int sa = 32 * rb + r, sc = 32 * ch + 16 * hf;
  f32x16 S = zero16();
  if (!STATES) {
    const float* s0 = A.P > 1 ? A.seg + (bh * A.P + p) * 4096 : (A.state ? A.state + bh * 4096 : nullptr);
    if (s0 && (A.P > 1 || !A.transposed)) {
#pragma unroll
      for (int x = 0; x < 16; x += 4) {
        const float4 f = *(const float4*)(s0 + sa * 64 + sc + x);
        S[x] = f.x, S[x + 1] = f.y, S[x + 2] = f.z, S[x + 3] = f.w;
      }
    } else if (s0) {
#pragma unroll
      for (int x = 0; x < 16; ++x) S[x] = s0[(sc + x) * 64 + sa];
    }
  }
  unsigned char* stile = lds + 2 * kTiles * kTile;
  auto put_state = [&](int buf) __attribute__((always_inline)) {
    u32x4 lo, hi;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      lo[x] = pack_bf16x2(S[2 * x], S[2 * x + 1]);
      hi[x] = pack_bf16x2(S[8 + 2 * x], S[9 + 2 * x]);
    }
    *(u32x4*)(stile + buf * kTile + toff(sa, sc / 8)) = lo;
    *(u32x4*)(stile + buf * kTile + toff(sa, sc / 8 + 1)) = hi;
  };

  // staging: thread tid moves granule tid % 8 of rows tid / 8 and 32 + tid / 8
  const int gr = tid & 7, r0 = tid >> 3;
  u32x4 gk[2], gv[2], qf[4], qn[4];
  auto load = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t at = row(c * kC + r0 + 32 * u) + 8 * gr;
      gk[u] = *(const u32x4*)(k + at);
      gv[u] = *(const u32x4*)(v + at);
    }
    if (!STATES) {
      const uint16_t* qr = q + row(c * kC + 32 * rb + r) + 8 * hf;
#pragma unroll
      for (int s = 0; s < 4; ++s) qn[s] = *(const u32x4*)(qr + 16 * s);
    }
  };
  const float ks = REV ? A.scale : 1.f;
  float wk[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) wk[u] = ks * decay_pow(g, (float)(kC - 1 + REV - (r0 + 32 * u)));
  auto stage = [&](int c, int buf) __attribute__((always_inline)) {
    unsigned char* t = lds + buf * kTiles * kTile;
    const int rem = len - c * kC;  // rows of this chunk
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int rr = r0 + 32 * u, at = toff(rr, gr);
      float w = wk[u];
      if (rem < kC) {
        w = rr < rem ? ks * decay_pow(g, (float)(rem - 1 + REV - rr)) : 0.f;
        if (rr >= rem) gk[u] = gv[u] = u32x4{0u, 0u, 0u, 0u};
      }
      u32x4 hi, lo;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = w * bf16_to_f32(gk[u][e] & 0xffffu), y = w * __uint_as_float(gk[u][e] & 0xffff0000u);
        hi[e] = pack_bf16x2(x, y);
        lo[e] = pack_bf16x2(x - bf16_to_f32(hi[e] & 0xffffu), y - __uint_as_float(hi[e] & 0xffff0000u));
      }
      *(u32x4*)(t + at) = gv[u];
      *(u32x4*)(t + kTile + at) = hi;
      *(u32x4*)(t + 2 * kTile + at) = lo;
      if (!STATES) *(u32x4*)(t + 3 * kTile + at) = gk[u];
    }
  };

  // transposing reads: lane 4 j + s of a block of 16 addresses row j
  const int bj = (lane >> 2) & 3, bs = lane & 3, bb = (lane >> 4) & 1;
  // columns 32 ch ..: permuted so that result row 8 (v / 4) + 4 hf + v % 4 is column 16 hf + v
  auto tr_perm = [&](const unsigned char* t, int rw) __attribute__((always_inline)) {
    return lds_tr16(t + toff(rw + bj, 4 * ch + 2 * (bs & 1) + bb) + 8 * (bs >> 1));
  };
  // columns 32 rb .. in order
  auto tr_nat = [&](const unsigned char* t, int rw) __attribute__((always_inline)) {
    return lds_tr16(t + toff(rw + bj, 4 * rb + 2 * bb + (bs >> 1)) + 8 * (bs & 1));
  };

  float wd[16], wo[16];
#pragma unroll
  for (int x = 0; x < 16; ++x) {
    const int d = r - (8 * (x / 4) + 4 * hf + x % 4);  // query minus key within a block
    wd[x] = d >= 0 ? A.scale * decay_pow(g, (float)d) : 0.f;
    wo[x] = A.scale * decay_pow(g, (float)(32 + d));
  }
  const float wi = (REV ? 1.f : A.scale) * decay_pow(g, (float)(32 * rb + r + 1 - REV));
  const float wc = decay_pow(g, (float)kC);

  if (c0 < c1) {
    load(c0);
    stage(c0, 0);
    if (!STATES) {
      put_state(0);
#pragma unroll
      for (int s = 0; s < 4; ++s) qf[s] = qn[s];
    }
    __syncthreads();
  }
  for (int c = c0; c < c1; ++c) {
    const int buf = (c - c0) & 1;
    const unsigned char* t = lds + buf * kTiles * kTile;
    const bool more = c + 1 < c1;
    if (more) load(c + 1);
    u32x4 vf[4];  // V^T: step x contracts tokens 16 x + {4 hf + 0..3, 8 + 4 hf + 0..3}
#pragma unroll
    for (int x = 0; x < 4; ++x) vf[x] = join(tr_perm(t, 16 * x + 4 * hf), tr_perm(t, 16 * x + 8 + 4 * hf));
    if (!STATES) {
      u32x4 pf[4];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        if (kb > rb) continue;
        f32x16 P = zero16();
#pragma unroll
        for (int s = 0; s < 4; ++s)
          P = mfma(*(const u32x4*)(t + 3 * kTile + toff(32 * kb + r, 2 * s + hf)), qf[s], P);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int x = 8 * u + 2 * e;
            pf[2 * kb + u][e] = kb == rb ? pack_bf16x2(P[x] * wd[x], P[x + 1] * wd[x + 1])
                                         : pack_bf16x2(P[x] * wo[x], P[x + 1] * wo[x + 1]);
          }
      }
      f32x16 o = zero16();
      const unsigned char* st = stile + buf * kTile;
#pragma unroll
      for (int s = 0; s < 4; ++s)
        o = mfma(join(tr_perm(st, 16 * s + 8 * hf), tr_perm(st, 16 * s + 8 * hf + 4)), qf[s], o);
#pragma unroll
      for (int x = 0; x < 16; ++x) o[x] *= wi;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (x / 2 <= rb) o = mfma(vf[x], pf[x], o);
      const int i = c * kC + 32 * rb + r;
      if (i < len) {
        const int64_t at = bh * A.n * 64 + row(i) + sc;
        if (A.out_f32) {
#pragma unroll
          for (int x = 0; x < 16; x += 4)
            *(float4*)((float*)A.out + at + x) = make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
        } else {
          u32x4 lo, hi;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            lo[x] = pack_bf16x2(o[2 * x], o[2 * x + 1]);
            hi[x] = pack_bf16x2(o[8 + 2 * x], o[9 + 2 * x]);
          }
          *(u32x4*)((uint16_t*)A.out + at) = lo;
          *(u32x4*)((uint16_t*)A.out + at + 8) = hi;
        }
      }
    }
    const float w = len - c * kC < kC ? decay_pow(g, (float)(len - c * kC)) : wc;
#pragma unroll
    for (int x = 0; x < 16; ++x) S[x] *= w;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int ra = 16 * x + 4 * hf;
      S = mfma(vf[x], join(tr_nat(t + kTile, ra), tr_nat(t + kTile, ra + 8)), S);
      S = mfma(vf[x], join(tr_nat(t + 2 * kTile, ra), tr_nat(t + 2 * kTile, ra + 8)), S);
    }
    if (more) {
      stage(c + 1, buf ^ 1);
      if (!STATES) {
        put_state(buf ^ 1);
#pragma unroll
        for (int s = 0; s < 4; ++s) qf[s] = qn[s];
      }
      __syncthreads();
    }
  }
  float* so = STATES ? A.seg + (bh * A.P + p) * 4096 : (p == A.P - 1 && A.state_out ? A.state_out + bh * 4096 : nullptr);
  if (so) {
#pragma unroll
    for (int x = 0; x < 16; x += 4)
      *(float4*)(so + sa * 64 + sc + x) = make_float4(S[x], S[x + 1], S[x + 2], S[x + 3]);
  }
  if (!STATES) {  // rows behind the sequence's end
    const int z0 = max(len, c0 * kC), z1 = p == A.P - 1 ? A.n : min(A.n, (c0 + A.cps) * kC);
    const int64_t base = (bh * A.n) * 64;
    if (A.out_f32) {
      for (int64_t x = (int64_t)z0 * 16 + tid; x < (int64_t)z1 * 16; x += 256)
        ((float4*)((float*)A.out + base))[x] = make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
      for (int64_t x = (int64_t)z0 * 8 + tid; x < (int64_t)z1 * 8; x += 256)
        ((u32x4*)((uint16_t*)A.out + base))[x] = u32x4{0u, 0u, 0u, 0u};
    }
  }
}

// Local states of the segments to the states before them, in place:
// s_0 = the initial state, s_{p+1} = l^(tokens of p) s_p + local_p.
__global__ __launch_bounds__(256) void k_lin_scan(float* seg, const float* state, const float* log_decay,
                                                  const int32_t* lengths, int H, int n, int P, int cps,
                                                  bool transposed) {
  const int64_t bh = blockIdx.x >> 4;
  const int e = (blockIdx.x & 15) * 256 + threadIdx.x;
  const float g = decay_log2(log_decay[bh % H]);
  const int len = length_of(lengths, bh / H, n);
  float s = !state ? 0.f : state[bh * 4096 + (transposed ? (e & 63) * 64 + (e >> 6) : e)];
  float* at = seg + bh * P * 4096 + e;
  for (int p0 = 0; p0 < P; p0 += 8) {
    float local[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) local[u] = p0 + u < P - 1 ? at[(int64_t)(p0 + u) * 4096] : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (p0 + u >= P) break;
      at[(int64_t)(p0 + u) * 4096] = s;
      const int64_t tokens = min((int64_t)max(len - (int64_t)(p0 + u) * cps * kC, (int64_t)0), (int64_t)cps * kC);
      s = fmaf(decay_pow(g, (float)tokens), s, local[u]);
    }
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

// Segments per slice and chunks per segment.
struct Split {
  int P, cps;
};
Split split_of(const LinearDims& d) {
  const int chunks = (d.n + kC - 1) / kC;
  const int64_t slices = (int64_t)d.B * d.H;
  // a launch of two workgroups per compute unit keeps HBM busy; a slice is
  // split where there are fewer than one each, since the segments' states cost
  // another pass over K and V
  int64_t P = slices >= 256 ? 1 : 512 / slices;
  if (P > chunks / 4) P = chunks / 4;
  if (P < 1) P = 1;
  const int cps = (int)((chunks + P - 1) / P);
  return Split{(chunks + cps - 1) / cps, cps};
}
size_t seg_bytes(const LinearDims& d) {
  const Split s = split_of(d);
  return s.P > 1 ? (size_t)d.B * d.H * s.P * 4096 * 4 : 0;
}

template <bool REV>
void chunked(const LinearDims& d, Chunked a, hipStream_t st) {
  const Split s = split_of(d);
  a.P = s.P;
  a.cps = s.cps;
  const unsigned slices = (unsigned)(d.B * d.H);
  if (s.P > 1) {
    {
      TimedLaunch tl("lin_states", st);
      hipLaunchKernelGGL((k_lin_chunk<REV, true>), dim3(slices * (s.P - 1)), dim3(256), 0, st, a);
    }
    TimedLaunch tl("lin_scan", st);
    hipLaunchKernelGGL(k_lin_scan, dim3(slices * 16), dim3(256), 0, st, a.seg, a.state, a.log_decay, a.lengths, d.H,
                       d.n, s.P, s.cps, a.transposed);
  }
  TimedLaunch tl("lin_chunk", st);
  hipLaunchKernelGGL((k_lin_chunk<REV, false>), dim3(slices * s.P), dim3(256), 0, st, a);
}

}  // namespace

size_t linear_workspace(const LinearDims& d) { return d.dtype == 1 ? seg_bytes(d) : 0; }

hipError_t launch_linear(const LinearDims& d, const void* Q, const void* K, const void* V, const float* log_decay,
                         const int32_t* lengths, const float* state, float scale, void* O, float* state_out, void* ws,
                         hipStream_t st) {
  if (d.dtype == 1) {
    Chunked a{(const uint16_t*)Q, (const uint16_t*)K, (const uint16_t*)V, false, true, true, log_decay, state, lengths,
              (float*)ws, state_out, O, d.H, d.Hk, d.n, 1, 1, scale, false, false};
    chunked<false>(d, a, st);
    return hipGetLastError();
  }
  walk(d, Walk{Q, K, V, false, true, true, log_decay, state, lengths, state_out, O, d.H, d.Hk, d.n, scale, false,
               false, false}, st);
  return hipGetLastError();
}

size_t linear_grad_workspace(const LinearDims& d) {
  return (d.H == d.Hk ? 0 : (size_t)d.B * d.H * d.n * 64 * 4) + (d.dtype == 1 ? seg_bytes(d) : 0);
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
  if (d.dtype == 1) {
    float* seg = (float*)((char*)ws + (grouped ? (size_t)d.B * d.H * d.n * 64 * 4 : 0));
    const uint16_t *q = (const uint16_t*)Q, *k = (const uint16_t*)K, *v = (const uint16_t*)V, *o = (const uint16_t*)dO;
    chunked<false>(d, Chunked{o, v, k, false, true, true, log_decay, state, lengths, seg, nullptr, dQ, d.H, d.Hk, d.n,
                              1, 1, scale, true, false}, st);
    chunked<true>(d, Chunked{v, o, q, true, false, false, log_decay, dstate, lengths, seg, nullptr, grouped ? ws : dK,
                             d.H, d.Hk, d.n, 1, 1, scale, true, grouped}, st);
    heads(dK);
    chunked<true>(d, Chunked{k, q, o, true, false, false, log_decay, dstate, lengths, seg, dstate_out,
                             grouped ? ws : dV, d.H, d.Hk, d.n, 1, 1, scale, false, grouped}, st);
    heads(dV);
    return hipGetLastError();
  }
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
