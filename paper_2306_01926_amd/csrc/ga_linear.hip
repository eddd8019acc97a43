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
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "ga_internal.h"

namespace ga {
namespace {

#include "ga_device.h"

// The decay of a state value over some tokens, l^n x.  Many decays in a row
// compound what the factor is off by, and 2^-24 of a factor near one is large
// against its distance to one; l^n - 1 is formed without that loss, and l^n x
// as x + (l^n - 1) x.  A small factor is exact enough as it is, and l^n - 1
// would not be.
struct Decay {
  float a, b;  // l^n = a + b with b 0 or 1
  __device__ __forceinline__ explicit Decay(float log_decay_n) {
    b = log_decay_n > -0.5f ? 1.f : 0.f;
    a = b != 0.f ? expm1f(log_decay_n) : expf(log_decay_n);
  }
  __device__ __forceinline__ float operator()(float x) const { return fmaf(a, x, b * x); }
};
// The same for a walk's equal chunks as one factor each: what the rounding of
// one is off by is taken from the next, so that their product is not.
struct Decays {
  Decay l;
  float off;
  __device__ __forceinline__ explicit Decays(float log_decay_n) : l(log_decay_n), off(0.f) {}
  __device__ __forceinline__ float next() {
    const float a = l.a + off, w = a + l.b;
    off = a - (w - l.b);
    return w;
  }
};

__device__ __forceinline__ int length_of(const int32_t* lengths, int64_t b, int n) {
  return lengths ? min(max(lengths[b], 0), n) : n;
}

// One token per sequence: 256 threads per slice, thread (r, g) holds rows
// r + 16 u of the state at columns 4 g .. 4 g + 3.  Bound by the state, 16 KB
// read and 16 KB written per slice (B H = 2048: 11.4 us, 5.9 TB/s; B H = 2: 2.4
// us); everything is fp32.
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
// group, in ascending order, rounded once.  Four values per thread.  grid.y: dV
// and dK, whose shares lie behind each other.  Bound by HBM (B H = 32, Hk = 2 of
// 8, n = 8000, bf16: 28 us for 147 MB).
template <class DT>
__global__ __launch_bounds__(256) void k_lin_heads(const float* __restrict__ part, int H, int Hk, int64_t row4,
                                                   int64_t total4, typename DT::T* __restrict__ dV,
                                                   typename DT::T* __restrict__ dK) {
  const int G = H / Hk;
  typename DT::T* out = blockIdx.y ? dK : dV;
  if (blockIdx.y) part += 4 * G * total4;
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
// all four products on the matrix cores.  A workgroup of eight waves walks the
// chunks of one slice, or of one of P segments of it: four waves form the
// output, 32 tokens by 32 value features each, four the state, a quadrant each
// in 16 registers, one chunk ahead of its use.
//
// Products are formed transposed (K Q^T, V^T P^T, ...), so the scores' result
// registers are the next product's operand as they are: no LDS round trip.
// The value rows feeding the last product are permuted so that a lane ends with
// 16 consecutive features of one token (32 bytes, stored from registers).
// K, V and Q rows sit in LDS as they come; the operands that need a column of
// them come from transposing LDS reads.
//
// B H = 128, n = 8000 (524 MB): 120 us, 4.4 TB/s, where a copy runs at 5.3; 160 us
// with four waves for both jobs and rows one chunk ahead.  A walk takes 0.8 us a
// chunk: the chain from one state to the next (conversion of the keys, an LDS
// round trip, the products) beside four waves of output; so few slices are bound
// by it, and are split, and many by HBM.
//
// Roundings: the scores after decay and the state that Q meets are rounded to
// bf16, as the matrix cores need (each term of an output passes one of the
// two); the state itself is fp32, and the decayed keys that it sums are kept
// as two bf16 parts (16 significant bits), two products each, or as three where
// the state is handed back: two leave it off by 2e-6 of its 2-norm.
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

// Byte offset of 16-byte granule q of row r of a tile of 128-byte rows.  The
// granule is XORed with a key of the row: rows two apart differ in its highest
// bit, so a transposing read's four rows of 64 bytes meet all 64 banks once,
// and eight rows of equal parity in all of it, as do 16 rows of one granule.
__device__ __forceinline__ int toff(int r, int q) {
  const int m = r >> 1;
  return r * 128 + ((q ^ (((m & 1) << 2) | (m & 2) | ((m >> 2) & 1))) << 4);
}
// A buffer of `bytes` bytes at p for loads and stores whose lanes beyond it read
// zeros and write nothing.  The walks below load and store without branches, so
// that the compiler can count what is in flight and wait for the oldest alone.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes, 0x00027000);
}
__device__ __forceinline__ u32x4 buf_load(Buffer b, int off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, off, 0, 0));
}
__device__ __forceinline__ void buf_store(Buffer b, int off, u32x4 x) {
  __builtin_amdgcn_raw_buffer_store_b128(x, b, off, 0, 0);
}

struct Chunked {
  const uint16_t *q, *k, *v, *w;                // roles (see the head of the file; w: the gradient's backward walk)
  bool q_shared, k_shared, v_shared, w_shared;  // the tensor has Hk heads
  const float *log_decay, *state;
  const int32_t* lengths;
  float* seg;        // [B H][P][64][64]: the segments' local states, or (scanned) the states before them; P > 1 only
  float* state_out;
  void *out, *out2;
  int H, Hk, n, P, cps;  // segments per slice, chunks per segment
  float scale;
  bool transposed, scanned;
};

// One segment of one slice, as its workgroup sees it.
// REV walks from a sequence's last token to its first; its state is R of the
// head of the file times l, the carry to the token before: a token's own decay
// is behind it, so the exponents are one lower at the output and one higher in
// the sum, and the scale sits in the sum.
template <bool REV>
struct Segment {
  const uint16_t *q, *k, *v, *w;
  int64_t bh;
  int p, len, c0, c1;
  float g, ld, ks;

  __device__ __forceinline__ Segment(const Chunked& A, int64_t slice, int segment) : bh(slice), p(segment) {
    const int h = (int)(bh % A.H);
    const int64_t b = bh / A.H, bk = b * A.Hk + h / (A.H / A.Hk);
    len = __builtin_amdgcn_readfirstlane(length_of(A.lengths, b, A.n));
    q = A.q + (A.q_shared ? bk : bh) * A.n * 64;
    k = A.k + (A.k_shared ? bk : bh) * A.n * 64;
    v = A.v + (A.v_shared ? bk : bh) * A.n * 64;
    w = A.w + (A.w_shared ? bk : bh) * A.n * 64;
    ld = fmaxf(A.log_decay[h], -1.0e30f);
    g = decay_log2(A.log_decay[h]);
    ks = REV ? A.scale : 1.f;
    c0 = p * A.cps;
    c1 = min(c0 + A.cps, (len + kC - 1) / kC);
  }
  // rows of chunk c (none behind the segment), the first one in memory, and
  // the place of walk row x among them (beyond them: out of the buffer)
  __device__ __forceinline__ int count(int c) const { return c < c1 ? min(len - c * kC, kC) : 0; }
  __device__ __forceinline__ int64_t first(int c, int nr) const {
    return REV ? (int64_t)len - (int64_t)c * kC - nr : (int64_t)c * kC;
  }
  __device__ __forceinline__ int place(int x, int nr) const { return REV ? nr - 1 - x : x; }
  // tokens of segment u
  __device__ __forceinline__ float tokens(const Chunked& A, int u) const {
    const int64_t t = (int64_t)A.cps * kC;
    return (float)min(max((int64_t)len - u * t, (int64_t)0), t);
  }
  // granule x of row rr of chunk c, decayed to the chunk's end, in bf16 parts
  template <int PARTS>
  __device__ __forceinline__ void decayed(u32x4 x, int rr, int c, u32x4 (&part)[PARTS]) const {
    // rows behind the end are zeros
    const float w = ks * decay_pow(g, (float)(max(count(c) - 1 - rr, 0) + REV));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float a = w * bf16_to_f32(x[e] & 0xffffu), b = w * __uint_as_float(x[e] & 0xffff0000u);
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        part[i][e] = pack_bf16x2(a, b);
        a -= bf16_to_f32(part[i][e] & 0xffffu);
        b -= __uint_as_float(part[i][e] & 0xffff0000u);
      }
    }
  }
  // the state's decay over chunk c (all but the last are whole)
  __device__ __forceinline__ float over(int c, Decays& whole) const {
    const int nr = count(c);
    return nr < kC ? decay_pow(g, (float)nr) : whole.next();
  }
  // Walks the segment's chunks: load(c, R) requests the rows of chunk c, three
  // chunks ahead of their use (HBM answers after about the time of two),
  // put(c, buf, R) puts them into a tile buffer, step(c, buf, R) computes chunk
  // c and puts the next chunk's rows R into the other buffer: one barrier a
  // chunk.  Three chunks a turn, as many sets of registers, and no way out
  // between them, which would cost copies of rows in flight (a wait for them).
  template <class Rows, class Load, class Put, class Step>
  __device__ __forceinline__ void walk(Load load, Put put, Step step) const {
    if (c0 >= c1) return;
    Rows R0, R1, R2;
    load(c0, R0);
    load(c0 + 1, R1);
    load(c0 + 2, R2);
    put(c0, 0, R0);
    __syncthreads();
    auto turn = [&](int c, int buf, const Rows& next, Rows& later) __attribute__((always_inline)) {
      load(c + 3, later);
      step(c, buf, next);
      __syncthreads();
    };
    int c = c0, buf = 0;
    for (; c + 3 <= c1; c += 3, buf ^= 1) {
      turn(c, buf, R1, R0);
      turn(c + 1, buf ^ 1, R2, R1);
      turn(c + 2, buf, R0, R2);
    }
    if (c < c1) turn(c, buf, R1, R0);
    if (c + 1 < c1) turn(c + 1, buf ^ 1, R2, R1);
  }
};

// Lane numbers of the operands: the transposing reads' row and 8-byte piece.
struct Lanes {
  int r, hf, bj, bs, bb;
  __device__ __forceinline__ explicit Lanes(int lane)
      : r(lane & 31), hf(lane >> 5), bj((lane >> 2) & 3), bs(lane & 3), bb((lane >> 4) & 1) {}
  // four rows from rw: columns 32 half .. in order, of a tile of 128-byte rows
  __device__ __forceinline__ u32x2 nat(const unsigned char* t, int rw, int half) const {
    return lds_tr16(t + toff(rw + bj, 4 * half + 2 * bb + (bs >> 1)) + 8 * (bs & 1));
  }
  // columns 32 half .. permuted so that result row 8 (v / 4) + 4 hf + v % 4 is column 16 hf + v
  __device__ __forceinline__ u32x2 perm(const unsigned char* t, int rw, int half) const {
    return lds_tr16(t + toff(rw + bj, 4 * half + 2 * (bs & 1) + bb) + 8 * (bs >> 1));
  }
};

// Features 32 half .. of 32 tokens from walk row x0, lane (r, hf) holding
// features 16 hf + 0..15 of token r, into the chunk's buffer.
template <bool OUT32, bool REV>
__device__ __forceinline__ void store_tokens(Buffer b, const Segment<REV>& G, int x0, int nr, int half, int lane,
                                             const f32x16& o) {
  if constexpr (OUT32) {
    const int off = (G.place(x0 + (lane & 31), nr) * 64 + 32 * half + 16 * (lane >> 5)) * 4;
#pragma unroll
    for (int x = 0; x < 16; x += 4)
      buf_store(b, off + 4 * x, u32x4{__float_as_uint(o[x]), __float_as_uint(o[x + 1]), __float_as_uint(o[x + 2]),
                                      __float_as_uint(o[x + 3])});
  } else {
    // lanes 16 apart exchange, so that four of them hold 64 bytes of one token
    u32x4 lo, hi;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const auto x = __builtin_amdgcn_permlane16_swap(pack_bf16x2(o[2 * e], o[2 * e + 1]),
                                                      pack_bf16x2(o[8 + 2 * e], o[9 + 2 * e]), false, false);
      lo[e] = x[0];
      hi[e] = x[1];
    }
    const int at = 64 * half + 16 * (lane >> 4);
    buf_store(b, G.place(x0 + (lane & 15), nr) * 128 + at, lo);
    buf_store(b, G.place(x0 + 16 + (lane & 15), nr) * 128 + at, hi);
  }
}

// A wave's operands for the update of its quadrant of the state (features 32 ah
// of the keys, 32 ch of the values): the value tile's columns and those of the
// decayed keys' parts, which lie behind each other.  Two chains of products run
// side by side, the first parts' into S, the others' into T.
template <int PARTS>
struct StateUpdate {
  u32x4 vf[4], kf[PARTS][4];  // step x contracts tokens 16 x + {4 hf + 0..3, 8 + 4 hf + 0..3}
  __device__ __forceinline__ StateUpdate(const unsigned char* values, const unsigned char* keys, const Lanes& L, int ah,
                                         int ch) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int ra = 16 * x + 4 * L.hf;
      vf[x] = join(L.perm(values, ra, ch), L.perm(values, ra + 8, ch));
#pragma unroll
      for (int i = 0; i < PARTS; ++i)
        kf[i][x] = join(L.nat(keys + i * kTile, ra, ah), L.nat(keys + i * kTile, ra + 8, ah));
    }
  }
  __device__ __forceinline__ void add(f32x16& S, f32x16& T) const {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      S = mfma(vf[x], kf[0][x], S);
#pragma unroll
      for (int i = 1; i < PARTS; ++i) T = mfma(vf[x], kf[i][x], T);
    }
  }
};

// The local states of the segments but the last, from zero: four waves, a
// quadrant of the state each.
template <bool REV, int PARTS>
__device__ __forceinline__ void local_states(const Chunked& A, unsigned char (*lds)[(1 + PARTS) * kTile]) {
  const int64_t bh = blockIdx.x / (A.P - 1);
  const Segment<REV> G(A, bh, (int)(blockIdx.x - bh * (A.P - 1)));
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Lanes L(tid & 63);
  const int ah = wave & 1, ch = wave >> 1, gr = tid & 7, r0 = tid >> 3;
  struct Rows {
    u32x4 k[2], v[2];
  };
  f32x16 S = zero16();
  Decays whole(G.ld * kC);
  auto put = [&](int c, int buf, const Rows& R) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u32x4 part[PARTS];
      G.decayed(R.k[u], r0 + 32 * u, c, part);
      const int at = toff(r0 + 32 * u, gr);
      *(u32x4*)(lds[buf] + at) = R.v[u];
#pragma unroll
      for (int i = 0; i < PARTS; ++i) *(u32x4*)(lds[buf] + (1 + i) * kTile + at) = part[i];
    }
  };
  G.template walk<Rows>(
      [&](int c, Rows& R) __attribute__((always_inline)) {
        const int nr = G.count(c);
        const Buffer bk = buffer(G.k + G.first(c, nr) * 64, nr * 128), bv = buffer(G.v + G.first(c, nr) * 64, nr * 128);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int off = G.place(r0 + 32 * u, nr) * 128 + 16 * gr;
          R.k[u] = buf_load(bk, off);
          R.v[u] = buf_load(bv, off);
        }
      },
      put,
      [&](int c, int buf, const Rows& next) __attribute__((always_inline)) {
        const unsigned char* t = lds[buf];
        const StateUpdate<PARTS> U(t, t + kTile, L, ah, ch);
        __builtin_amdgcn_sched_barrier(0);
        const float w = G.over(c, whole);
#pragma unroll
        for (int x = 0; x < 16; ++x) S[x] *= w;
        f32x16 T = zero16();
        U.add(S, T);
        put(c + 1, buf ^ 1, next);
#pragma unroll
        for (int x = 0; x < 16; ++x) S[x] += T[x];
      });
  float* so = A.seg + (bh * A.P + G.p) * 4096 + (32 * ah + L.r) * 64 + 32 * ch + 16 * L.hf;
#pragma unroll
  for (int x = 0; x < 16; x += 4) *(float4*)(so + x) = make_float4(S[x], S[x + 1], S[x + 2], S[x + 3]);
}

// grid (slices (P - 1), directions): a gradient needs the states of both walks.
template <int PARTS>
__global__ __launch_bounds__(256, PARTS == 2 ? 3 : 2) void k_lin_states(Chunked F, Chunked B) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[2][(1 + PARTS) * kTile];  // V, the decayed K's parts
  if (blockIdx.y == 0)
    local_states<false, PARTS>(F, lds);
  else
    local_states<true, PARTS>(B, lds);
}

// Outputs of a forward walk (and the final state): workgroup `block` of slices P.
// B H = 8, n = 100003: the states' pass over K and V 49 us (4.2 TB/s), the scan 7,
// this 76 (5.4 TB/s).
constexpr int forward_buf(int PARTS) { return (4 + PARTS) * kTile; }  // V, the state, Q, K, the decayed K's parts
template <int PARTS>
__device__ __forceinline__ void forward_walk(const Chunked& A, int block, unsigned char (*lds)[forward_buf(PARTS)]) {
  const int64_t bh = block / A.P;
  const Segment<false> G(A, bh, (int)(block - bh * A.P));
  // the wave's index is scalar, so that branches on it are jumps: matrix
  // instructions do not heed the lane mask
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const Lanes L(lane);
  constexpr int kV = 0, kS = kTile, kQ = 2 * kTile, kK = 3 * kTile;
  const int ch = (wave >> 1) & 1;

  auto put_key = [&](int buf, int row, int gr, u32x4 k, const u32x4(&part)[PARTS]) __attribute__((always_inline)) {
    unsigned char* t = lds[buf] + kK + toff(row, gr);
    *(u32x4*)t = k;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) *(u32x4*)(t + (1 + i) * kTile) = part[i];
  };

  if (wave >= 4) {
    // the state S[a][c], a = 32 ah + r, c = 32 ch + 16 hf + 0..15; its waves
    // also bring the values and the first 32 keys: granule tid % 8
    const int ah = wave & 1, sa = 32 * ah + L.r, sc = 32 * ch + 16 * L.hf, gr = tid & 7, r0 = (tid >> 3) & 31;
    struct Rows {
      u32x4 k, v[2];
    };
    f32x16 S = zero16();
    const bool given = A.state && !A.scanned;
    if (A.scanned || (given && !A.transposed)) {
      const float* s0 = (A.scanned ? A.seg + (bh * A.P + G.p) * 4096 : A.state + bh * 4096) + sa * 64 + sc;
#pragma unroll
      for (int x = 0; x < 16; ++x) S[x] = s0[x];
    } else if (given) {
#pragma unroll
      for (int x = 0; x < 16; ++x) S[x] = A.state[bh * 4096 + (sc + x) * 64 + sa];
    }
    if (!A.scanned) {
      for (int u = 0; u < G.p; ++u) {
        const float w = decay_pow(G.g, G.tokens(A, u));
        const float* s0 = A.seg + (bh * A.P + u) * 4096 + sa * 64 + sc;
#pragma unroll
        for (int x = 0; x < 16; ++x) S[x] = fmaf(w, S[x], s0[x]);
      }
    }
    u32x4 part[PARTS];
    Decays whole(G.ld * kC);
    auto put = [&](int buf, const Rows& R) __attribute__((always_inline)) {
      put_key(buf, r0, gr, R.k, part);
#pragma unroll
      for (int u = 0; u < 2; ++u) *(u32x4*)(lds[buf] + kV + toff(r0 + 32 * u, gr)) = R.v[u];
    };
    auto put_state = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < 16; x += 8)
        *(u32x4*)(lds[buf] + kS + toff(sa, 4 * ch + 2 * L.hf + x / 8)) =
            u32x4{pack_bf16x2(S[x], S[x + 1]), pack_bf16x2(S[x + 2], S[x + 3]), pack_bf16x2(S[x + 4], S[x + 5]),
                  pack_bf16x2(S[x + 6], S[x + 7])};
    };
    G.template walk<Rows>(
        [&](int c, Rows& R) __attribute__((always_inline)) {
          const int nr = G.count(c);
          const Buffer bk = buffer(G.k + G.first(c, nr) * 64, nr * 128), bv = buffer(G.v + G.first(c, nr) * 64, nr * 128);
          R.k = buf_load(bk, G.place(r0, nr) * 128 + 16 * gr);
#pragma unroll
          for (int u = 0; u < 2; ++u) R.v[u] = buf_load(bv, G.place(r0 + 32 * u, nr) * 128 + 16 * gr);
        },
        [&](int c, int buf, const Rows& R) __attribute__((always_inline)) {
          G.decayed(R.k, r0, c, part);
          put(buf, R);
          put_state(buf);
        },
        [&](int c, int buf, const Rows& next) __attribute__((always_inline)) {
          const unsigned char* t = lds[buf];
          // the conversion comes first: the output's waves have the LDS then
          G.decayed(next.k, r0, c + 1, part);
          const float w = G.over(c, whole);
#pragma unroll
          for (int x = 0; x < 16; ++x) S[x] *= w;
          f32x16 T = zero16();
          __builtin_amdgcn_sched_barrier(0);
          const StateUpdate<PARTS> U(t + kV, t + kK + kTile, L, ah, ch);
          U.add(S, T);
          __builtin_amdgcn_sched_group_barrier(0x100, 8 + 4 * PARTS - 4, 0);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x8, PARTS, 0);
            if (x < 2) __builtin_amdgcn_sched_group_barrier(0x100, 2 + 2 * PARTS, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
          put(buf ^ 1, next);
#pragma unroll
          for (int x = 0; x < 16; ++x) S[x] += T[x];
          put_state(buf ^ 1);
        });
    if (G.p == A.P - 1 && A.state_out) {
      float* so = A.state_out + bh * 4096 + sa * 64 + sc;
#pragma unroll
      for (int x = 0; x < 16; x += 4) *(float4*)(so + x) = make_float4(S[x], S[x + 1], S[x + 2], S[x + 3]);
    }
  } else {
    float wd[16], wo[16];  // decays inside a block of 32 tokens, and between two
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const int d = L.r - (8 * (x / 4) + 4 * L.hf + x % 4);  // query minus key within a block
      wd[x] = d >= 0 ? A.scale * decay_pow(G.g, (float)d) : 0.f;
      wo[x] = A.scale * decay_pow(G.g, (float)(32 + d));
    }
    unsigned char* out = (unsigned char*)A.out + bh * A.n * 128;
    // rows that these waves bring, by their 128 threads each: the shorter
    // block's the last 32 keys, the longer block's the queries
    const int gr = lane & 7, r0 = (lane >> 3) + 8 * ch;
    // the second block of tokens meets two blocks of keys, the first one: a
    // loop for each, without branches
    auto outputs = [&](auto block) __attribute__((always_inline)) {
      constexpr int RB = decltype(block)::value;
      const float wi = A.scale * decay_pow(G.g, (float)(32 * RB + L.r + 1));
      constexpr int kRows = RB ? 4 : 2;
      struct Rows {
        u32x4 x[kRows];
      };
      u32x4 part[2][PARTS];
      auto convert = [&](int c, const Rows& R) __attribute__((always_inline)) {
        if constexpr (RB == 0) {
#pragma unroll
          for (int u = 0; u < 2; ++u) G.decayed(R.x[u], 32 + r0 + 16 * u, c, part[u]);
        }
      };
      auto put = [&](int buf, const Rows& R) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
          if constexpr (RB == 0)
            put_key(buf, 32 + r0 + 16 * u, gr, R.x[u], part[u]);
          else
            *(u32x4*)(lds[buf] + kQ + toff(r0 + 16 * u, gr)) = R.x[u];
        }
      };
      G.template walk<Rows>(
          [&](int c, Rows& R) __attribute__((always_inline)) {
            const int nr = G.count(c);
            const Buffer b = buffer((RB ? G.q : G.k) + G.first(c, nr) * 64, nr * 128);
#pragma unroll
            for (int u = 0; u < kRows; ++u)
              R.x[u] = buf_load(b, G.place((RB ? 0 : 32) + r0 + 16 * u, nr) * 128 + 16 * gr);
          },
          [&](int c, int buf, const Rows& R) __attribute__((always_inline)) {
            convert(c, R);
            put(buf, R);
          },
          [&](int c, int buf, const Rows& next) __attribute__((always_inline)) {
            const unsigned char* t = lds[buf];
            u32x4 qf[4], kf[RB + 1][4], sf[4], vf[2 * RB + 2], pf[2 * RB + 2];
#pragma unroll
            for (int s = 0; s < 4; ++s) qf[s] = *(const u32x4*)(t + kQ + toff(32 * RB + L.r, 2 * s + L.hf));
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
              for (int kb = 0; kb <= RB; ++kb) kf[kb][s] = *(const u32x4*)(t + kK + toff(32 * kb + L.r, 2 * s + L.hf));
#pragma unroll
            for (int s = 0; s < 4; ++s)
              sf[s] = join(L.perm(t + kS, 16 * s + 8 * L.hf, ch), L.perm(t + kS, 16 * s + 8 * L.hf + 4, ch));
#pragma unroll
            for (int x = 0; x < 2 * RB + 2; ++x)
              vf[x] = join(L.perm(t + kV, 16 * x + 4 * L.hf, ch), L.perm(t + kV, 16 * x + 8 + 4 * L.hf, ch));
            f32x16 P[RB + 1], o = zero16(), oi = zero16();
#pragma unroll
            for (int kb = 0; kb <= RB; ++kb) P[kb] = zero16();
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
              for (int kb = 0; kb <= RB; ++kb) P[kb] = mfma(kf[kb][s], qf[s], P[kb]);
#pragma unroll
            for (int s = 0; s < 4; ++s) oi = mfma(sf[s], qf[s], oi);
            // reads of the keys, then the products with reads of the rest between
            __builtin_amdgcn_sched_group_barrier(0x100, 4 * RB + 12, 0);
#pragma unroll
            for (int x = 0; x < 4 * RB + 4; ++x) {
              __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
              __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x8, 4, 0);
            __builtin_amdgcn_sched_barrier(0);
            convert(c + 1, next);
#pragma unroll
            for (int u = 0; u < 2 * RB + 2; ++u)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int x = 8 * (u & 1) + 2 * e;
                const float* w = u / 2 == RB ? wd : wo;
                pf[u][e] = pack_bf16x2(P[u / 2][x] * w[x], P[u / 2][x + 1] * w[x + 1]);
              }
#pragma unroll
            for (int x = 0; x < 2 * RB + 2; ++x) o = mfma(vf[x], pf[x], o);
#pragma unroll
            for (int x = 0; x < 16; ++x) o[x] = fmaf(wi, oi[x], o[x]);
            const int nr = G.count(c);
            const Buffer bo = buffer(out + G.first(c, nr) * 128, nr * 128);
            store_tokens<false>(bo, G, 32 * RB, nr, ch, lane, o);
            put(buf ^ 1, next);
          });
    };
    if ((wave & 1) == 0)
      outputs(std::integral_constant<int, 0>{});
    else
      outputs(std::integral_constant<int, 1>{});
    // rows behind the sequence's end, by the output's 256 threads
    const int z0 = max(G.len, G.c0 * kC), z1 = G.p == A.P - 1 ? A.n : min(A.n, (G.c0 + A.cps) * kC);
    for (int64_t x = (int64_t)z0 * 8 + tid; x < (int64_t)z1 * 8; x += 256) ((u32x4*)out)[x] = u32x4{0u, 0u, 0u, 0u};
  }
}

// The gradients of K and V in one backward walk: dV has the roles q = K, k = Q,
// v = dO, dK the roles q = V (w), k = dO, v = Q, and both meet the same state
// R[a][c] (a: feature of q and k, c: of v and dO), dK with its other side.
// Eight waves: waves 0-3 form 32 tokens by 64 features of dV (0, 1) or dK
// (2, 3), waves 4-7 the state.  out: dV, out2: dK; OUT32: they are fp32 (a
// query head's share of a shared head's gradient).  Both walks of the gradient
// together are bound by HBM: they read seven tensors, the states' pass four, and
// write three (B H = 32, n = 20000: 65 + 147 us, 5.4 TB/s; B H = 128, n = 8000, not
// split: 257 us, 5.1 TB/s).
constexpr int backward_buf(int PARTS) { return (5 + PARTS) * kTile; }  // dO, K, V, the state, Q, the decayed Q's parts
template <bool OUT32, int PARTS>
__device__ __forceinline__ void backward_walk(const Chunked& A, int block, unsigned char (*lds)[backward_buf(PARTS)]) {
  constexpr int kO = 0, kK = kTile, kV = 2 * kTile, kS = 3 * kTile, kQ = 4 * kTile;
  const int64_t bh = block / A.P;
  const Segment<true> G(A, bh, (int)(block - bh * A.P));
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const Lanes L(lane);

  // every thread brings granule tid % 8 of row tid / 8 of the four tensors
  struct Rows {
    u32x4 k, v, q, w;
  };
  const int gr = tid & 7, r0 = tid >> 3, at = toff(r0, gr);
  u32x4 part[PARTS];
  auto load = [&](int c, Rows& R) __attribute__((always_inline)) {
    const int nr = G.count(c);
    const int64_t f = G.first(c, nr) * 64;
    const int off = G.place(r0, nr) * 128 + 16 * gr;
    R.k = buf_load(buffer(G.k + f, nr * 128), off);
    R.v = buf_load(buffer(G.v + f, nr * 128), off);
    R.q = buf_load(buffer(G.q + f, nr * 128), off);
    R.w = buf_load(buffer(G.w + f, nr * 128), off);
  };
  auto put = [&](int buf, const Rows& R) __attribute__((always_inline)) {
    unsigned char* t = lds[buf] + at;
    *(u32x4*)(t + kQ) = R.k;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) *(u32x4*)(t + kQ + (1 + i) * kTile) = part[i];
    *(u32x4*)(t + kO) = R.v;
    *(u32x4*)(t + kK) = R.q;
    *(u32x4*)(t + kV) = R.w;
  };

  if (wave >= 4) {
    const int ah = wave & 1, ch = (wave >> 1) & 1, sa = 32 * ah + L.r, sc = 32 * ch + 16 * L.hf;
    f32x16 S = zero16();
    Decays whole(G.ld * kC);
    const float* s0 = A.scanned ? A.seg + (bh * A.P + G.p) * 4096 : (A.state ? A.state + bh * 4096 : nullptr);
    if (s0) {
#pragma unroll
      for (int x = 0; x < 16; ++x) S[x] = s0[sa * 64 + sc + x];
    }
    if (!A.scanned) {
      for (int u = 0; u < G.p; ++u) {
        const float w = decay_pow(G.g, G.tokens(A, u));
        const float* s1 = A.seg + (bh * A.P + u) * 4096 + sa * 64 + sc;
#pragma unroll
        for (int x = 0; x < 16; ++x) S[x] = fmaf(w, S[x], s1[x]);
      }
    }
    auto put_state = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < 16; x += 8)
        *(u32x4*)(lds[buf] + kS + toff(sa, 4 * ch + 2 * L.hf + x / 8)) =
            u32x4{pack_bf16x2(S[x], S[x + 1]), pack_bf16x2(S[x + 2], S[x + 3]), pack_bf16x2(S[x + 4], S[x + 5]),
                  pack_bf16x2(S[x + 6], S[x + 7])};
    };
    G.template walk<Rows>(
        load,
        [&](int c, int buf, const Rows& R) __attribute__((always_inline)) {
          G.decayed(R.k, r0, c, part);
          put(buf, R);
          put_state(buf);
        },
        [&](int c, int buf, const Rows& next) __attribute__((always_inline)) {
          const unsigned char* t = lds[buf];
          G.decayed(next.k, r0, c + 1, part);
          const float w = G.over(c, whole);
#pragma unroll
          for (int x = 0; x < 16; ++x) S[x] *= w;
          f32x16 T = zero16();
          __builtin_amdgcn_sched_barrier(0);
          const StateUpdate<PARTS> U(t + kO, t + kQ + kTile, L, ah, ch);
          U.add(S, T);
          put(buf ^ 1, next);
#pragma unroll
          for (int x = 0; x < 16; ++x) S[x] += T[x];
          put_state(buf ^ 1);
        });
    if (G.p == A.P - 1 && A.state_out) {
      float* so = A.state_out + bh * 4096 + sa * 64 + sc;
#pragma unroll
      for (int x = 0; x < 16; x += 4) *(float4*)(so + x) = make_float4(S[x], S[x + 1], S[x + 2], S[x + 3]);
    }
  } else {
    float wd[16], wo[16];  // decays inside a block of 32 tokens, and between two
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const int d = L.r - (8 * (x / 4) + 4 * L.hf + x % 4);
      wd[x] = d >= 0 ? A.scale * decay_pow(G.g, (float)d) : 0.f;
      wo[x] = A.scale * decay_pow(G.g, (float)(32 + d));
    }
    const bool keys = wave >= 2;  // dK
    const int tq = keys ? kV : kK, tk = keys ? kO : kQ, tv = keys ? kQ : kO;
    constexpr int kEl = OUT32 ? 4 : 2;
    unsigned char* out = (unsigned char*)(keys ? A.out2 : A.out) + bh * A.n * (64 * kEl);
    // row of the state whose features a are the result's rows, permuted as L.perm does
    const int prow = 16 * ((L.r >> 2) & 1) + 4 * (L.r >> 3) + (L.r & 3);
    auto outputs = [&](auto block) __attribute__((always_inline)) {
      constexpr int RB = decltype(block)::value;
      const float wi = decay_pow(G.g, (float)(32 * RB + L.r));
      G.template walk<Rows>(
          load,
          [&](int c, int buf, const Rows& R) __attribute__((always_inline)) {
            G.decayed(R.k, r0, c, part);
            put(buf, R);
          },
          [&](int c, int buf, const Rows& next) __attribute__((always_inline)) {
            const unsigned char* t = lds[buf];
            u32x4 qf[4], pf[2 * RB + 2];
#pragma unroll
            for (int s = 0; s < 4; ++s) qf[s] = *(const u32x4*)(t + tq + toff(32 * RB + L.r, 2 * s + L.hf));
            f32x16 P[RB + 1], o[2] = {zero16(), zero16()};
#pragma unroll
            for (int kb = 0; kb <= RB; ++kb) P[kb] = zero16();
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
              for (int kb = 0; kb <= RB; ++kb)
                P[kb] = mfma(*(const u32x4*)(t + tk + toff(32 * kb + L.r, 2 * s + L.hf)), qf[s], P[kb]);
            if (keys) {
#pragma unroll
              for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  o[e] = mfma(*(const u32x4*)(t + kS + toff(32 * e + prow, 2 * s + L.hf)), qf[s], o[e]);
            } else {
#pragma unroll
              for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  o[e] = mfma(join(L.perm(t + kS, 16 * s + 8 * L.hf, e), L.perm(t + kS, 16 * s + 8 * L.hf + 4, e)),
                              qf[s], o[e]);
            }
            G.decayed(next.k, r0, c + 1, part);
#pragma unroll
            for (int u = 0; u < 2 * RB + 2; ++u)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int x = 8 * (u & 1) + 2 * e;
                const float* w = u / 2 == RB ? wd : wo;
                pf[u][e] = pack_bf16x2(P[u / 2][x] * w[x], P[u / 2][x + 1] * w[x + 1]);
              }
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
              for (int x = 0; x < 16; ++x) o[e][x] *= wi;
#pragma unroll
            for (int x = 0; x < 2 * RB + 2; ++x)
#pragma unroll
              for (int e = 0; e < 2; ++e)
                o[e] = mfma(join(L.perm(t + tv, 16 * x + 4 * L.hf, e), L.perm(t + tv, 16 * x + 8 + 4 * L.hf, e)), pf[x],
                            o[e]);
            put(buf ^ 1, next);
            const int nr = G.count(c);
            const Buffer bo = buffer(out + G.first(c, nr) * (64 * kEl), nr * 64 * kEl);
#pragma unroll
            for (int e = 0; e < 2; ++e) store_tokens<OUT32>(bo, G, 32 * RB, nr, e, lane, o[e]);
          });
    };
    if ((wave & 1) == 0)
      outputs(std::integral_constant<int, 0>{});
    else
      outputs(std::integral_constant<int, 1>{});
    // rows behind the sequence's end, by the 128 threads of each output
    const int z0 = max(G.len, G.c0 * kC), z1 = G.p == A.P - 1 ? A.n : min(A.n, (G.c0 + A.cps) * kC);
    constexpr int kG = 64 * kEl / 16;  // 16-byte granules per row
    for (int64_t x = (int64_t)z0 * kG + (tid & 127); x < (int64_t)z1 * kG; x += 128)
      ((u32x4*)out)[x] = u32x4{0u, 0u, 0u, 0u};
  }
}

// grid: slices P.  PARTS: 3 where the final state is handed back.
template <int PARTS>
__global__ __launch_bounds__(512, 2) void k_lin_forward(Chunked A) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[2][forward_buf(PARTS)];
  forward_walk<PARTS>(A, blockIdx.x, lds);
}

// dQ (the forward walk F) and dK, dV (the backward walk B) side by side: they
// share no result, and one launch of both fills the compute units where one of
// them would not.  grid: slices (B.P + F.P), the longer backward walks first.
// PARTS: 3 where the initial state's gradient is handed back.
template <bool OUT32, int PARTS>
__global__ __launch_bounds__(512, 2) void k_lin_backward(Chunked F, Chunked B, int backward) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[2 * backward_buf(PARTS)];
  static_assert(forward_buf(2) <= backward_buf(PARTS), "the forward walk's tiles fit");
  if ((int)blockIdx.x < backward)
    backward_walk<OUT32, PARTS>(B, blockIdx.x, (unsigned char(*)[backward_buf(PARTS)])lds);
  else
    forward_walk<2>(F, blockIdx.x - backward, (unsigned char(*)[forward_buf(2)])lds);
}

// Local states of the segments to the states before them, in place:
// s_0 = the initial state, s_{p+1} = l^(tokens of p) s_p + local_p.
// grid (slices 16, directions).
struct Scan {
  float* seg;
  const float *state, *log_decay;
  const int32_t* lengths;
  int H, n, P, tokens;  // tokens per segment
  bool transposed, wanted;
};
__global__ __launch_bounds__(256) void k_lin_scan(Scan F, Scan B) {
  const Scan& A = blockIdx.y == 0 ? F : B;
  if (!A.wanted) return;
  const int64_t bh = blockIdx.x >> 4;
  const int e = (blockIdx.x & 15) * 256 + threadIdx.x;
  const float ld = fmaxf(A.log_decay[bh % A.H], -1.0e30f);
  const Decay whole(ld * A.tokens);
  const int len = length_of(A.lengths, bh / A.H, A.n);
  float s = !A.state ? 0.f : A.state[bh * 4096 + (A.transposed ? (e & 63) * 64 + (e >> 6) : e)];
  float* at = A.seg + bh * A.P * 4096 + e;
  for (int p0 = 0; p0 < A.P; p0 += 8) {
    float local[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) local[u] = p0 + u < A.P - 1 ? at[(int64_t)(p0 + u) * 4096] : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (p0 + u >= A.P) break;
      at[(int64_t)(p0 + u) * 4096] = s;
      const int64_t tokens = min(max((int64_t)len - (int64_t)(p0 + u) * A.tokens, (int64_t)0), (int64_t)A.tokens);
      s = (tokens == A.tokens ? whole : Decay(ld * tokens))(s) + local[u];
    }
  }
}

// ---------------------------------------------------------------- fp32, by chunks
//
// The same by chunks of 32 tokens, every operand as three bf16 parts and every
// product as six (24 bits; the fp32 matrix instructions take 64 cycles for two
// features where the six take 192 for sixteen).  A register that holds a result
// is an operand of the next product in any of the roles that the walk needs.
// With (r, hf) the lane and j(x) = 8 (x / 4) + 4 hf + x % 4 for x = 0..15:
//   lane r holds K[r][j(x)], Q[r][j(x)] (features j(x) and 32 + j(x)),
//   V[j(x)][r] (tokens j(x)), S[j(x)][r] (features of k), scores^T[j(x)][r],
//   O^T[j(x)][r],
// eight of which in order are the contracted values of one product.  Only the
// keys, needed by column for the state, pass through LDS; the decay to the
// chunk's end is on the values there.  A wave walks a segment for one half of
// the value features without a barrier; a workgroup is the halves of two
// segments.
// A chunk takes 3.2 us: 84 matrix instructions of 32 cycles and 900 of the VALU
// that make the parts, one after the other for the most part (3.6 us with the
// fp32 instructions, 112 of 64 cycles).  B H = 24, n = 1111, gradient: 47 us, 51
// with those.  Rows of a later chunk are requested where the registers of this
// one's become free, hundreds of cycles before their use.
constexpr int kC32 = 32;

struct Walk32 {
  const float *q, *k, *v;             // roles (see the head of the file)
  bool q_shared, k_shared, v_shared;  // the tensor has Hk heads
  const float *log_decay, *state;
  const int32_t* lengths;
  float *seg, *state_out, *out;  // seg: [B H][P][64][64], local states or (outputs) the states before each segment
  int H, Hk, n, P, tokens;       // segments per slice, tokens per segment (a multiple of 32)
  float scale;
  bool transposed;  // the state and seg are S^T in this walk's roles
};

// Eight fp32 values as three bf16 parts each (24 significant bits; exact but for
// values below 2^-110, whose last bits lie below the type's range, and above
// 3.38e38, which round to infinity), and the six products of parts that 24 bits
// of a product need (what is left out is 2^-24 of it).
struct Split8 {
  u32x4 p[3];
};
template <class F>
__device__ __forceinline__ Split8 split8(F value) {
  Split8 s;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float a = value(2 * e), b = value(2 * e + 1);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      s.p[i][e] = pack_bf16x2(a, b);
      a -= __uint_as_float(s.p[i][e] << 16);
      b -= __uint_as_float(s.p[i][e] & 0xffff0000u);
    }
  }
  return s;
}
__device__ __forceinline__ f32x16 mfma6(const Split8& a, const Split8& b, f32x16 c) {
  c = mfma(a.p[2], b.p[0], c);
  c = mfma(a.p[0], b.p[2], c);
  c = mfma(a.p[1], b.p[1], c);
  c = mfma(a.p[1], b.p[0], c);
  c = mfma(a.p[0], b.p[1], c);
  return mfma(a.p[0], b.p[0], c);
}
__device__ __forceinline__ float buf_load1(Buffer b, int off) {
  return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b, off, 0, 0));
}

constexpr int kPart32 = kC32 * 128;  // bytes of a chunk's keys, one part
constexpr int kLds32 = 3 * kPart32;  // of a wave

// Segments 2 block and 2 block + 1 of `items` in all (STATES: without each slice's last).
template <bool REV, bool STATES>
__device__ __forceinline__ void walk32(const Walk32& A, int block, int items, unsigned char (*lds)[kLds32]) {
  const int nseg = STATES ? A.P - 1 : A.P;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), item = 2 * block + (wave >> 1);
  if (item >= items) return;  // (no barriers)
  const int64_t bh = item / nseg;
  const int p = (int)(item - bh * nseg), h = (int)(bh % A.H);
  const int64_t b = bh / A.H, bk = b * A.Hk + h / (A.H / A.Hk);
  const int len = __builtin_amdgcn_readfirstlane(length_of(A.lengths, b, A.n));
  const int lane = threadIdx.x & 63, r = lane & 31, hf = lane >> 5;
  const int ch = wave & 1;
  unsigned char* kt = lds[wave];  // the keys' parts, a token a row
  const Lanes L(lane);
  const float* q = A.q + (A.q_shared ? bk : bh) * A.n * 64;
  const float* k = A.k + (A.k_shared ? bk : bh) * A.n * 64;
  const float* v = A.v + (A.v_shared ? bk : bh) * A.n * 64 + 32 * ch;
  float* out = A.out + bh * A.n * 64 + 32 * ch;
  const float g = decay_log2(A.log_decay[h]);
  const float ks = REV ? A.scale : 1.f;
  Decays whole(fmaxf(A.log_decay[h], -1.0e30f) * kC32);
  const int64_t t0 = (int64_t)p * A.tokens, t1 = min(t0 + A.tokens, (int64_t)len);
  auto jx = [&](int x) __attribute__((always_inline)) { return 8 * (x / 4) + 4 * hf + x % 4; };

  // Rows of the chunk at walk position t.  Their buffer starts with the first of
  // them in memory; rows behind the end are outside of it (v and out start 32 ch
  // features into a row, so theirs ends as much behind the last one, where no
  // lane reaches).
  auto count = [&](int64_t t) __attribute__((always_inline)) { return (int)min(max(t1 - t, (int64_t)0), (int64_t)kC32); };
  auto rows = [&](const float* base, int64_t t, int nr) __attribute__((always_inline)) {
    return buffer(base + (REV ? (int64_t)len - t - nr : t) * 64, nr * 256);
  };
  auto place = [&](int x, int nr) __attribute__((always_inline)) { return REV ? nr - 1 - x : x; };

  float qa[32], ka[32], vc[16];
  auto load_row = [&](const float* base, int64_t t, float(&x)[32]) __attribute__((always_inline)) {
    const int nr = count(t), off = place(r, nr) * 256 + 16 * hf;
    const Buffer bf = rows(base, t, nr);
#pragma unroll
    for (int u = 0; u < 8; ++u) {  // features 8 u + 4 hf + 0..3
      const u32x4 y = buf_load(bf, off + 32 * u);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * u + e] = __uint_as_float(y[e]);
    }
  };
  auto load_values = [&](int64_t t) __attribute__((always_inline)) {
    const int nr = count(t);
    const Buffer bv = rows(v, t, nr);
#pragma unroll
    for (int x = 0; x < 16; ++x) vc[x] = buf_load1(bv, place(jx(x), nr) * 256 + 4 * r);
  };
  f32x16 S[2] = {zero16(), zero16()};  // S[32 e + j(x)][32 ch + r]
  if (!STATES) {
    const float* s0 = A.P > 1 ? A.seg + (bh * A.P + p) * 4096 : (A.state ? A.state + bh * 4096 : nullptr);
    if (s0 && A.transposed) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int x = 0; x < 16; ++x) S[e][x] = s0[(32 * ch + r) * 64 + 32 * e + jx(x)];
    } else if (s0) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int x = 0; x < 16; ++x) S[e][x] = s0[(32 * e + jx(x)) * 64 + 32 * ch + r];
    }
  }
  float wd[16];
#pragma unroll
  for (int x = 0; x < 16; ++x) wd[x] = r >= jx(x) ? A.scale * decay_pow(g, (float)(r - jx(x))) : 0.f;
  const float wi = (REV ? 1.f : A.scale) * decay_pow(g, (float)(r + 1 - REV));

  // decay of each value row to the chunk's end
  float wv[16];
  auto to_end = [&](int nr) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 16; ++x) wv[x] = ks * decay_pow(g, (float)(max(nr - 1 - jx(x), 0) + REV));
  };
  to_end(kC32);

  if (t0 < t1) {
    load_row(k, t0, ka);
    if (!STATES) load_row(q, t0, qa);
    load_values(t0);
  }
  for (int64_t t = t0; t < t1; t += kC32) {
    const int nr = count(t);
    if (nr < kC32) to_end(nr);  // (the last chunk; rows behind the end are zeros)
    f32x16 P = zero16();
    Split8 qp[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const Split8 kp = split8([&](int e) { return ka[8 * s + e]; });
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        *(u32x2*)(kt + i * kPart32 + toff(r, 2 * s) + 8 * hf) = u32x2{kp.p[i][0], kp.p[i][1]};
        *(u32x2*)(kt + i * kPart32 + toff(r, 2 * s + 1) + 8 * hf) = u32x2{kp.p[i][2], kp.p[i][3]};
      }
      if (!STATES) {
        qp[s] = split8([&](int e) { return qa[8 * s + e]; });
        P = mfma6(kp, qp[s], P);
      }
    }
    load_row(k, t + kC32, ka);
    __builtin_amdgcn_sched_barrier(0);  // (or the compiler requests everything at the end)
    if (!STATES) {
      f32x16 oi = zero16(), o = zero16();
#pragma unroll
      for (int s = 0; s < 4; ++s)
        oi = mfma6(split8([&](int e) { return S[s / 2][8 * (s % 2) + e]; }), qp[s], oi);
      load_row(q, t + kC32, qa);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        o = mfma6(split8([&](int e) { return vc[8 * u + e]; }),
                  split8([&](int e) { return P[8 * u + e] * wd[8 * u + e]; }), o);
      const Buffer bo = rows(out, t, nr);
      const int row = place(r, nr) * 256 + 16 * hf;
#pragma unroll
      for (int x = 0; x < 16; x += 4) {
        u32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = __float_as_uint(fmaf(wi, oi[x + e], o[x + e]));
        buf_store(bo, row + 8 * x, y);
      }
    }
    const float w = nr < kC32 ? decay_pow(g, (float)nr) : whole.next();
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int x = 0; x < 16; ++x) S[e][x] *= w;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const Split8 vd = split8([&](int e) { return vc[8 * u + e] * wv[8 * u + e]; });
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        Split8 kf;
#pragma unroll
        for (int i = 0; i < 3; ++i)
          kf.p[i] = join(L.nat(kt + i * kPart32, 16 * u + 4 * hf, e), L.nat(kt + i * kPart32, 16 * u + 8 + 4 * hf, e));
        S[e] = mfma6(kf, vd, S[e]);
      }
    }
    load_values(t + kC32);
    __builtin_amdgcn_sched_barrier(0);
  }
  float* so = STATES ? A.seg + (bh * A.P + p) * 4096
                     : (p == A.P - 1 && A.state_out ? A.state_out + bh * 4096 : nullptr);
  if (so) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int x = 0; x < 16; ++x) so[(32 * e + jx(x)) * 64 + 32 * ch + r] = S[e][x];
  }
  if (!STATES) {  // rows behind the sequence's end
    const int64_t z1 = p == A.P - 1 ? (int64_t)A.n : min((int64_t)A.n, t0 + A.tokens);
    for (int64_t t = max((int64_t)len, t0) + (lane >> 3); t < z1; t += 8)
      *(float4*)(out + t * 64 + 4 * (lane & 7)) = make_float4(0.f, 0.f, 0.f, 0.f);
  }
}

// grid (segments but each slice's last / 2, directions): the local states of forward and backward walks.
__global__ __launch_bounds__(256, 1) void k_lin_states_f32(Walk32 F, Walk32 B, int items) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[4][kLds32];
  if (blockIdx.y == 0)
    walk32<false, true>(F, blockIdx.x, items, lds);
  else
    walk32<true, true>(B, blockIdx.x, items, lds);
}
// grid segments / 2.
__global__ __launch_bounds__(256, 2) void k_lin_forward_f32(Walk32 A, int items) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[4][kLds32];
  walk32<false, false>(A, blockIdx.x, items, lds);
}
// grid (segments / 2, walks): dQ, dK, dV from walk `from` on.
__global__ __launch_bounds__(256, 2) void k_lin_backward_f32(Walk32 Q, Walk32 K, Walk32 V, int from, int items) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[4][kLds32];
  const int walk = from + blockIdx.y;
  if (walk == 0)
    walk32<false, false>(Q, blockIdx.x, items, lds);
  else
    walk32<true, false>(walk == 1 ? K : V, blockIdx.x, items, lds);
}

// Segments per slice and chunks per segment.
struct Split {
  int P, cps;
};
// The number of segments with the least expected time, in us, among those whose
// workgroups fit the GPU at once.  A walk is bound by the latency of its chunks
// (0.8 us a chunk forward, 1.4 times that in the gradient's pair of walks) or by
// HBM; segments take a launch and half a walk more for their states, and read
// two of the tensors (four) again.  Measured, whole against split: B H = 128, n =
// 8000: 120 and 137 us (two); B H = 32, n = 20000: 284 and 95 (eight); B H = 64, n
// = 1024: 17.8 and 19.3 (four); B H = 2, n = 1024: 16.9 and 13.5 (eight).
Split split_of(const LinearDims& d, int walks) {
  const int chunks = (d.n + kC - 1) / kC;
  const int64_t all = (int64_t)d.B * d.H * walks;
  const double slow = walks == 1 ? 1.0 : 1.4, tensor = (double)d.B * d.H * d.n * 128 / 5.3e6;  // us of one tensor
  Split best{1, chunks};
  double least = 0;
  for (int64_t P = 1; P == 1 || P * all <= 256;) {
    const int cps = (int)((chunks + P - 1) / P);
    const double full = fmin((double)(P * all) / 256, 1);
    const double walk = P == 1 ? 4.4 + cps * slow * (0.8 + 0.08 * full)
                               : 7.6 + 3.7 * full + (P <= 8 ? 0.45 * P : 3.5 + 0.12 * P) +
                                     cps * slow * (1.2 + 0.35 * full);
    const double bytes = tensor * (walks == 1 ? (P == 1 ? 4 : 6) : (P == 1 ? 10 : 14));
    const double us = fmax(walk, bytes) + 0.1 * walk;
    if (P == 1 || us < least) best = Split{(int)P, cps}, least = us;
    if (cps == 1) break;
    P = (chunks + cps - 2) / (cps - 1);  // the fewest segments of fewer chunks
  }
  return best;
}
size_t seg_bytes(const LinearDims& d, Split s) {
  return s.P > 1 ? (size_t)d.B * d.H * s.P * 4096 * 4 : 0;
}

void set_split(Chunked& a, Split s) {
  a.P = s.P;
  a.cps = s.cps;
  // (an initial state that is updated in place is read before any workgroup writes it)
  a.scanned = s.P > 8 || (s.P > 1 && a.state && a.state == a.state_out);
}

// The states before the segments of one walk, or of the two of a gradient.
// exact: a state is handed back.
void segment_states(const LinearDims& d, const Chunked& f, const Chunked& b, unsigned directions, bool exact,
                    hipStream_t st) {
  const unsigned slices = (unsigned)(d.B * d.H);
  if (f.P > 1) {
    TimedLaunch tl("lin_states", st);
    const dim3 grid(slices * (f.P - 1), directions);
    if (exact)
      hipLaunchKernelGGL(k_lin_states<3>, grid, dim3(256), 0, st, f, b);
    else
      hipLaunchKernelGGL(k_lin_states<2>, grid, dim3(256), 0, st, f, b);
  }
  if (f.scanned || b.scanned) {
    TimedLaunch tl("lin_scan", st);
    auto scan = [](const Chunked& c) {
      return Scan{c.seg, c.state, c.log_decay, c.lengths, c.H, c.n, c.P, c.cps * kC, c.transposed, c.scanned};
    };
    hipLaunchKernelGGL(k_lin_scan, dim3(slices * 16, directions), dim3(256), 0, st, scan(f), scan(b));
  }
}

// fp32, in the same way: a slice's two halves are a wave each, and 1024 waves, one
// a SIMD, are a round (two waves a SIMD take nearly twice as long as one).  A
// chunk of 64 tokens takes a walk 6.1 us and the states' pass 2.0, more where all
// SIMDs work.  Measured, whole against split: B H = 16, n = 1024: 102 and 25 us (16
// segments); gradient, B H = 64, n = 256: 33 and 36 (two), n = 4096: 425 and 268
// (eight); B H = 128, n = 1024: 117 and 134 (four).
Split split32_of(const LinearDims& d, int walks) {
  const int chunks = (d.n + kC - 1) / kC;
  const double waves = 2.0 * d.B * d.H / 1024;
  const auto rounds = [](double w) { return w <= 1 ? 1 : 0.5 * (w + ceil(w)); };
  Split best{1, chunks};
  double least = 0;
  for (int P = 1; P == 1 || P * waves * walks <= 6;) {
    const int cps = (chunks + P - 1) / P;
    const double main = P * waves * walks, before = P * waves * (walks == 1 ? 1 : 2);
    const double us = P == 1 ? 4 + cps * rounds(main) * (6.1 + 0.7 * fmin(main, 1))
                             : 11.4 + 0.13 * P + cps * (rounds(main) * (6.1 + 0.7 * fmin(main, 1)) +
                                                        rounds(before) * (2.0 + 3.2 * fmin(before, 1)));
    if (P == 1 || us < least) best = Split{P, cps}, least = us;
    if (cps == 1) break;
    P = (chunks + cps - 2) / (cps - 1);
  }
  return best;
}

Walk32 walk32_of(const LinearDims& d, Split s, const float* log_decay, const int32_t* lengths, float scale) {
  Walk32 a{};
  a.log_decay = log_decay, a.lengths = lengths, a.scale = scale;
  a.H = d.H, a.Hk = d.Hk, a.n = d.n, a.P = s.P, a.tokens = s.cps * kC;
  return a;
}

void segment_states32(const LinearDims& d, const Walk32& f, const Walk32& b, unsigned directions, hipStream_t st) {
  if (f.P < 2) return;
  const unsigned slices = (unsigned)(d.B * d.H);
  {
    TimedLaunch tl("lin_states", st);
    const int items = (int)slices * (f.P - 1);
    hipLaunchKernelGGL(k_lin_states_f32, dim3((items + 1) / 2, directions), dim3(256), 0, st, f, b, items);
  }
  auto scan = [](const Walk32& c) {
    return Scan{c.seg, c.state, c.log_decay, c.lengths, c.H, c.n, c.P, c.tokens, false, true};
  };
  TimedLaunch tl("lin_scan", st);
  hipLaunchKernelGGL(k_lin_scan, dim3(slices * 16, directions), dim3(256), 0, st, scan(f), scan(b));
}

}  // namespace

size_t linear_workspace(const LinearDims& d) {
  return seg_bytes(d, d.dtype == 1 ? split_of(d, 1) : split32_of(d, 1));
}

hipError_t launch_linear(const LinearDims& d, const void* Q, const void* K, const void* V, const float* log_decay,
                         const int32_t* lengths, const float* state, float scale, void* O, float* state_out, void* ws,
                         hipStream_t st) {
  if (d.dtype == 1) {
    Chunked a{};
    a.q = (const uint16_t*)Q, a.k = (const uint16_t*)K, a.v = (const uint16_t*)V;
    a.k_shared = a.v_shared = true;
    a.log_decay = log_decay, a.state = state, a.lengths = lengths;
    a.seg = (float*)ws, a.state_out = state_out, a.out = O;
    a.H = d.H, a.Hk = d.Hk, a.n = d.n, a.scale = scale;
    set_split(a, split_of(d, 1));
    segment_states(d, a, Chunked{}, 1, state_out != nullptr, st);
    TimedLaunch tl("lin_forward", st);
    const dim3 wgs((unsigned)(d.B * d.H * a.P));
    if (state_out)
      hipLaunchKernelGGL(k_lin_forward<3>, wgs, dim3(512), 0, st, a);
    else
      hipLaunchKernelGGL(k_lin_forward<2>, wgs, dim3(512), 0, st, a);
    return hipGetLastError();
  }
  Walk32 a = walk32_of(d, split32_of(d, 1), log_decay, lengths, scale);
  a.q = (const float*)Q, a.k = (const float*)K, a.v = (const float*)V;
  a.k_shared = a.v_shared = true;
  a.state = state, a.seg = (float*)ws, a.state_out = state_out, a.out = (float*)O;
  segment_states32(d, a, Walk32{}, 1, st);
  TimedLaunch tl("lin_forward", st);
  const int items = d.B * d.H * a.P;
  hipLaunchKernelGGL(k_lin_forward_f32, dim3((items + 1) / 2), dim3(256), 0, st, a, items);
  return hipGetLastError();
}

size_t linear_grad_workspace(const LinearDims& d) {
  // a query head's shares of shared dK and dV, and the states before both walks' segments
  const size_t part = d.H == d.Hk ? 0 : (size_t)d.B * d.H * d.n * 64 * 4;
  return 2 * part + 2 * seg_bytes(d, d.dtype == 1 ? split_of(d, 2) : split32_of(d, 3));
}

hipError_t launch_linear_grad(const LinearDims& d, const void* Q, const void* K, const void* V, const void* dO,
                              const float* log_decay, const int32_t* lengths, const float* state, const float* dstate,
                              float scale, void* dQ, void* dK, void* dV, float* dstate_out, void* ws, hipStream_t st) {
  const bool grouped = d.H != d.Hk;
  const size_t part = grouped ? (size_t)d.B * d.H * d.n * 64 * 4 : 0;
  const int64_t row4 = (int64_t)d.n * 16, total4 = (int64_t)d.B * d.Hk * row4;
  const unsigned grid = (unsigned)((total4 + 255) / 256 < 8192 ? (total4 + 255) / 256 : 8192);
  auto heads = [&]() {
    if (!grouped) return;
    TimedLaunch tl("lin_heads", st);
    if (d.dtype == 1)
      hipLaunchKernelGGL(k_lin_heads<BF16>, dim3(grid, 2), dim3(256), 0, st, (const float*)ws, d.H, d.Hk, row4, total4,
                         (uint16_t*)dV, (uint16_t*)dK);
    else
      hipLaunchKernelGGL(k_lin_heads<F32>, dim3(grid, 2), dim3(256), 0, st, (const float*)ws, d.H, d.Hk, row4, total4,
                         (float*)dV, (float*)dK);
  };
  if (d.dtype == 1) {
    Chunked a{};
    a.log_decay = log_decay, a.lengths = lengths, a.seg = (float*)((char*)ws + 2 * part);
    a.H = d.H, a.Hk = d.Hk, a.n = d.n, a.scale = scale;
    Chunked b = a;
    a.q = (const uint16_t*)dO, a.k = (const uint16_t*)V, a.v = (const uint16_t*)K;
    a.k_shared = a.v_shared = true;
    a.state = state, a.transposed = true, a.out = dQ;
    b.q = (const uint16_t*)K, b.k = (const uint16_t*)Q, b.v = (const uint16_t*)dO, b.w = (const uint16_t*)V;
    b.q_shared = b.w_shared = true;
    b.state = dstate, b.state_out = dstate_out;
    b.out = grouped ? ws : dV, b.out2 = grouped ? (char*)ws + part : dK;
    const Split s = split_of(d, 2);
    b.seg = a.seg + seg_bytes(d, s) / 4;
    set_split(a, s);
    set_split(b, s);
    segment_states(d, a, b, 2, dstate_out != nullptr, st);
    {
      TimedLaunch tl("lin_backward", st);
      const int half = d.B * d.H * s.P;
      const dim3 wgs((unsigned)(2 * half));
#define GA_LIN_BACKWARD(OUT32, PARTS) \
  hipLaunchKernelGGL((k_lin_backward<OUT32, PARTS>), wgs, dim3(512), 0, st, a, b, half)
      if (dstate_out) {
        if (grouped) GA_LIN_BACKWARD(true, 3);
        else GA_LIN_BACKWARD(false, 3);
      } else {
        if (grouped) GA_LIN_BACKWARD(true, 2);
        else GA_LIN_BACKWARD(false, 2);
      }
#undef GA_LIN_BACKWARD
    }
    heads();
    return hipGetLastError();
  }
  const Split s = split32_of(d, 3);
  // the states of both directions, S[k feature][v feature] and R[q feature][dO feature]
  Walk32 f = walk32_of(d, s, log_decay, lengths, scale), r = f;
  f.k = (const float*)K, f.v = (const float*)V, f.k_shared = f.v_shared = true;
  f.q = (const float*)Q, r.q = (const float*)K;
  r.k = (const float*)Q, r.v = (const float*)dO, r.q_shared = true;
  f.seg = (float*)((char*)ws + 2 * part), r.seg = f.seg + seg_bytes(d, s) / 4;
  f.state = state, r.state = dstate;
  segment_states32(d, f, r, 2, st);
  Walk32 dq = f, dv = r, dk = r;
  dq.q = (const float*)dO, dq.k = (const float*)V, dq.v = (const float*)K, dq.transposed = true, dq.out = (float*)dQ;
  dv.out = grouped ? (float*)ws : (float*)dV, dv.state_out = dstate_out;
  dk.q = (const float*)V, dk.k = (const float*)dO, dk.v = (const float*)Q, dk.transposed = true;
  dk.out = grouped ? (float*)((char*)ws + part) : (float*)dK;
  {
    TimedLaunch tl("lin_backward", st);
    const int items = d.B * d.H * s.P, wgs = (items + 1) / 2;
    // a final state's gradient that is updated in place by dV's walk is read by dK's first
    const bool apart = s.P == 1 && dstate && dstate == dstate_out;
    hipLaunchKernelGGL(k_lin_backward_f32, dim3(wgs, apart ? 2 : 3), dim3(256), 0, st, dq, dk, dv, 0, items);
    if (apart) hipLaunchKernelGGL(k_lin_backward_f32, dim3(wgs, 1), dim3(256), 0, st, dq, dk, dv, 2, items);
  }
  heads();
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
