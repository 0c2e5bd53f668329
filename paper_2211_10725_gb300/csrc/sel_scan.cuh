// Shared by the selective-scan kernels and their entry points.
//
//   s = softplus(delta + bias),  x = s u,  a_t = exp(s A)
//   h_t = a_t h_{t-1} + x_t B_t,   y_t = (sum_n C_t h_t + D u_t) silu(z_t)
//
// A thread holds NS states (4, 8, 12 or 16) of two neighbouring channels of a group (a
// pair), in pairs of floats: v[2 k + j] is the states 2 k and 2 k + 1 of channel j, and one
// instruction serves both.  (B and C come in such pairs from where they lie; with the
// channels paired instead, what B or C enters took two instructions.)  P threads side by side (1,
// 2 or 4, P NS >= N) hold a pair's states, so that a warp has 32 / P pairs, and share out its
// tokens where inputs are made ready and results finished.  A warp works alone: B and C
// of a few tokens lie in shared memory of its own, and no barrier joins it to another
// warp.  Shared memory gives an SM 32 words a clock, however many lanes read the
// same one: a multiply-add that takes its operand from there has to serve several states or
// channels.
// The decay of a span of tokens is exp(A sum s), so a cut axis hands on one sum a
// channel beside the states.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "launch.cuh"
#include "scan_host.cuh"
#include "snn.h"
#include "snn_device.cuh"

namespace snn {
namespace sscan {

constexpr int kMaxN = 64;
constexpr int kTile = 8;          // tokens between checkpoints
constexpr int kSettle = 16;       // tokens between settle()s, whole tiles
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct Seq {  // [B, T, channels]
  void* data = nullptr;
  int64_t sb = 0, st = 0;
};
struct Mat {  // [B, T, G, N]
  void* data = nullptr;
  int64_t sb = 0, st = 0, sg = 0;
};

struct Args {
  int B, T, D, N, G, Dg;   // Dg channels of a group
  int softplus;
  int pair_ok;             // channel pairs lie on their own boundaries in every tensor
  int quads;               // so do fours of states of B and C
  int pairs;               // of a group
  int N2;                  // twos of states
  int spans, span;         // cuts of the axis, tokens of each
  int fine, span_fine;     // parts of a span of which the ends are found, tokens of each
  Seq u, delta, z, y, gy, gu, gdelta, gz;
  Mat Bm, Cm;
  const float *A, *D_skip, *bias;
  const int32_t *seq_lens, *slots;
  const float* state_in;
  float* state_out;
  int64_t num_slots;
  float* ckpt;             // [B][ceil(T / 8)][G][N2][pairs][4]: two states of one channel, then the other
  float* ends;             // [spans fine][B][G][N2][pairs][4]: what a part adds to the state
  float2* sums;            // [spans fine][B][G pairs]: of s over a part
  // backward
  const float* grad_state_out;
  float* grad_state_in;
  float *part_B, *part_C;  // [blocks of a group][B][T][G][N]
  float* part_A;           // [spans][B][D][N]
  float *part_D, *part_bias;  // [spans][B][D]
};

__device__ __forceinline__ int seq_len(const Args& g, int b) {
  if (!g.seq_lens) return g.T;
  const int n = g.seq_lens[b];
  return n < 0 ? 0 : (n > g.T ? g.T : n);
}

__device__ __forceinline__ float ex2(float x) {
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(x));
  return x;
}
// A channel's value, for both of its states.
__device__ __forceinline__ float2 of_channel(float2 v, int j) { return f2(j & 1 ? v.y : v.x); }
__device__ __forceinline__ float2 across(float2 a, float2 b) { return make_float2(a.x + a.y, b.x + b.y); }
__device__ __forceinline__ float2 ex2(float2 x) { return make_float2(ex2(x.x), ex2(x.y)); }
__device__ __forceinline__ float rcp(float x) {
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(x));
  return x;
}
__device__ __forceinline__ float2 rcp(float2 x) { return make_float2(rcp(x.x), rcp(x.y)); }
__device__ __forceinline__ float2 root(float2 x) {
  asm("sqrt.approx.ftz.f32 %0, %0;" : "+f"(x.x));
  asm("sqrt.approx.ftz.f32 %0, %0;" : "+f"(x.y));
  return x;
}

// softplus and its slope.  With e = e^-|x|: log(1 + e^x) = max(x, 0) + log(1 + e), and
// log(1 + e) = 2 atanh(r), r = e / (2 + e) <= 1/3.  The area tangent's series r + r^3 (1/3 + q / 5 +
// q^2 / 7 + ...), q = r^2 <= 1/9, with the bracket as the cubic that fits it there (Chebyshev): off by
// a quarter of 2^-24.  The slope is 1 / (1 + e) or e / (1 + e).  For fp32 inputs e gets back what
// the product |x| log2(e) was rounded by, |x| 2^-25 of it.  From |x| = 128 on, where e is zero
// (its power is flushed), |x| stays there: past 2.36e38 the product would be infinite and the rest of its
// rounding no number, with x = -inf, whose s is zero, among them.  A NaN stays one.
__device__ __forceinline__ float at_most_128(float x) {
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(128.0f));
  return x;
}
template <typename T>
__device__ __forceinline__ float2 softplus(float2 x, float2* slope) {
  constexpr float kLog2ELow = 1.92596303e-8f;
  float2 a = make_float2(-fabsf(x.x), -fabsf(x.y));
  if constexpr (sizeof(T) == 4) a = make_float2(-at_most_128(fabsf(x.x)), -at_most_128(fabsf(x.y)));
  const float2 t = mul2(a, f2(kLog2E));
  float2 e = ex2(t);
  if constexpr (sizeof(T) == 4) {
    const float2 rest = fma2(a, f2(kLog2ELow), fma2(a, f2(kLog2E), make_float2(-t.x, -t.y)));
    e = fma2(e, mul2(rest, f2(kLn2)), e);
  }
  const float2 r = mul2(e, rcp(add2(e, f2(2.0f)))), q = mul2(r, r);
  float2 p = fma2(q, f2(0.13433774f), f2(0.14116979f));
  p = fma2(p, q, f2(0.20003836f));
  p = fma2(p, q, f2(0.33333319f));
  p = fma2(mul2(p, q), r, r);
  if (slope) {
    const float2 one = rcp(add2(e, f2(1.0f)));
    *slope = mul2(make_float2(x.x >= 0.0f ? 1.0f : e.x, x.y >= 0.0f ? 1.0f : e.y), one);
  }
  return fma2(f2(2.0f), p, make_float2(fmaxf(x.x, 0.0f), fmaxf(x.y, 0.0f)));
}

// A state over a part of the axis that adds e to it, s the sum of the part's steps.  Large steps can
// add up past fp32; that sum stays finite, as the infinite one times an A of zero (that of
// a state that is absent, too) is no number.  The power is taken as the square of its root, at most
// 2^127: a growing state's (of a negative sum) can be past fp32 while the state is not, and
// so zero stays zero and a state becomes infinite where its value is past fp32.  (No branch: the
// next part's loads go past it; with one, 777 tokens of 1001 channels took 28 us for 23.)
template <int NS>
__device__ __forceinline__ void join(float2 (&h)[NS], const float2 (&A2)[NS], float2 s, const float2 (&e)[NS]) {
  constexpr float kMost = 3.402823466e38f;
  s = mul2(make_float2(fminf(fmaxf(s.x, -kMost), kMost), fminf(fmaxf(s.y, -kMost), kMost)), f2(0.5f));
#pragma unroll
  for (int q = 0; q < NS; ++q) {
    const float2 t = mul2(of_channel(s, q), A2[q]);
    const float2 root = ex2(make_float2(fminf(t.x, 127.0f), fminf(t.y, 127.0f)));
    h[q] = fma2(root, mul2(root, h[q]), e[q]);
  }
}

// The approximate power of two of an argument t below zero is low on average (measured, of arguments with
// all their bits): by 0.11 units of 2^-24 up to |t| = 0.002, by 0.4 from 0.008 to 1/2.  A state
// that remembers a thousand tokens multiplies a thousand of them.  The 0.11 units are a larger t
// (one of zero still gives exactly one); what is left, about 0.33 min(|t| / 0.0082, 1)^2 units, goes back
// into the states for kSettle tokens at a time: 0.33 min((|A| / 0.0082)^2 sum s^2, n) units, n = (sum s)^2 / sum s^2
// the number of tokens that the sum consists of: all of equal steps, one where one step stands
// among steps near zero.
constexpr float kLift = 0.11f / 16777216.0f / kLn2, kCap = 0.0082f, kUnits = 0.33f / 16777216.0f;
struct alignas(16) Steps {
  float2 sum = {0.0f, 0.0f}, squares = {0.0f, 0.0f};
  __device__ __forceinline__ void add(float2 s) {
    sum = add2(sum, s);
    squares = fma2(s, s, squares);
  }
  __device__ __forceinline__ void add(const Steps& o) {
    sum = add2(sum, o.sum);
    squares = add2(squares, o.squares);
  }
};
template <int NS>
__device__ __forceinline__ void settle(float2 (&h)[NS], const float2 (&A2)[NS], const Steps& s) {
  constexpr float kMost = kSettle;
  // (n of no steps, and of steps past fp32, is no number: kMost)
  const float2 n = mul2(mul2(s.sum, s.sum), rcp(s.squares)), by = root(mul2(s.squares, f2(kUnits / (kCap * kCap))));
  const float2 most = mul2(make_float2(fminf(n.x, kMost), fminf(n.y, kMost)), f2(kUnits));
#pragma unroll
  for (int q = 0; q < NS; ++q) {
    const float2 of = mul2(A2[q], of_channel(by, q)), part = mul2(of, of);
    const float cap = q & 1 ? most.y : most.x;
    h[q] = fma2(make_float2(fminf(part.x, cap), fminf(part.y, cap)), h[q], h[q]);
  }
}

// 1 / (1 + e^-x).  Results rounded to 16 bits take the approximate power of
// two and reciprocal: the rounding of x log2(e) costs |x| 2^-24 of the result.
template <typename T>
__device__ __forceinline__ float sigmoid(float x) {
  if constexpr (sizeof(T) == 4) return __frcp_rn(1.0f + expf(-x));
  else return rcp(1.0f + ex2(-kLog2E * x));
}
template <typename T>
__device__ __forceinline__ float2 sigmoid(float2 x) {
  if constexpr (sizeof(T) == 4) return make_float2(sigmoid<T>(x.x), sigmoid<T>(x.y));
  else return rcp(add2(ex2(mul2(x, f2(-kLog2E))), f2(1.0f)));
}

// The channels c and c + 1 of a token as they lie in memory.
template <typename T>
struct Raw {
  uint32_t w[sizeof(T) / 2];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = 0;
  }
  __device__ __forceinline__ void load(const T* p, bool pair, bool second) {
    if (pair) {
      if constexpr (sizeof(T) == 2) {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
      } else {
        const uint2 a = *reinterpret_cast<const uint2*>(p);
        w[0] = a.x;
        w[1] = a.y;
      }
    } else if constexpr (sizeof(T) == 2) {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
      w[0] = h[0] | (second ? (uint32_t)h[1] << 16 : 0u);
    } else {
      const uint32_t* h = reinterpret_cast<const uint32_t*>(p);
      w[0] = h[0];
      w[1] = second ? h[1] : 0u;
    }
  }
  __device__ __forceinline__ float2 get() const {
    if constexpr (sizeof(T) == 2) return Elem<T>::to2(w[0]);
    else return make_float2(__uint_as_float(w[0]), __uint_as_float(w[1]));
  }
};

template <typename T>
__device__ __forceinline__ void put_pair(T* p, float2 v, bool pair, bool second) {
  if (pair) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t*>(p) = Elem<T>::from2(v.x, v.y);
    else *reinterpret_cast<float2*>(p) = v;
  } else {
    Elem<T>::store1(p, v.x);
    if (second) Elem<T>::store1(p + 1, v.y);
  }
}

// s of the two channels of a delta with its bias, and its slope (if asked for).
template <typename T>
__device__ __forceinline__ float2 step_of(float2 raw, bool soft, float2* slope = nullptr) {
  if (soft) return softplus<T>(raw, slope);
  if (slope) *slope = f2(1.0f);
  return raw;
}

// A thread's states of its pair in an fp32 [.., D, N] array, from channel 0's row on;
// absent states are zero.
template <int NS>
__device__ __forceinline__ void load_states(const float* p, int N, int n0, bool second, float2 (&v)[NS]) {
  if (N % 4 == 0) {
#pragma unroll
    for (int q = 0; q < NS; q += 4) {
      float a[4] = {0.0f, 0.0f, 0.0f, 0.0f}, b[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (n0 + q < N) {
        Elem<float>::load4(p + n0 + q, a);
        if (second) Elem<float>::load4(p + N + n0 + q, b);
      }
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        v[q + i] = make_float2(a[i], a[i + 1]);
        v[q + i + 1] = make_float2(b[i], b[i + 1]);
      }
    }
  } else {
#pragma unroll
    for (int q = 0; q < NS; q += 2) {
      const bool in = n0 + q < N, in2 = n0 + q + 1 < N;
      v[q] = make_float2(in ? p[n0 + q] : 0.0f, in2 ? p[n0 + q + 1] : 0.0f);
      v[q + 1] = make_float2(in && second ? p[N + n0 + q] : 0.0f, in2 && second ? p[N + n0 + q + 1] : 0.0f);
    }
  }
}
template <int NS>
__device__ __forceinline__ void store_states(float* p, int N, int n0, bool second, const float2 (&v)[NS]) {
#pragma unroll
  for (int q = 0; q < NS; q += 2) {
    if (n0 + q < N) {
      p[n0 + q] = v[q].x;
      if (second) p[N + n0 + q] = v[q + 1].x;
    }
    if (n0 + q + 1 < N) {
      p[n0 + q + 1] = v[q].y;
      if (second) p[N + n0 + q + 1] = v[q + 1].y;
    }
  }
}

// The same in [N2][pairs][4] arrays (ends, checkpoints): p at the pair, n0 even.
template <int NS>
__device__ __forceinline__ void load_twos(const float* p, const Args& g, int n0, float2 (&v)[NS]) {
#pragma unroll
  for (int q = 0; q < NS; q += 2) {
    float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int k = (n0 + q) >> 1;
    if (k < g.N2) Elem<float>::load4(p + (int64_t)k * g.pairs * 4, a);
    v[q] = make_float2(a[0], a[1]);
    v[q + 1] = make_float2(a[2], a[3]);
  }
}
template <int NS>
__device__ __forceinline__ void store_twos(float* p, const Args& g, int n0, const float2 (&v)[NS]) {
#pragma unroll
  for (int q = 0; q < NS; q += 2) {
    const int k = (n0 + q) >> 1;
    const float a[4] = {v[q].x, v[q].y, v[q + 1].x, v[q + 1].y};
    if (k < g.N2) Elem<float>::store4(p + (int64_t)k * g.pairs * 4, a);
  }
}

// Four states (n0 ..) of B or C of a token as they lie in memory; zero for absent ones.
template <typename T>
struct Four {
  uint32_t w[sizeof(T)];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) w[i] = 0;
  }
  __device__ __forceinline__ void load(const T* p, bool quads, int absent) {  // absent: of the four
    if (quads) {
      if constexpr (sizeof(T) == 2) {
        const uint2 a = *reinterpret_cast<const uint2*>(p);
        w[0] = a.x, w[1] = a.y;
      } else {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q < 4 - absent) {
          if constexpr (sizeof(T) == 2) w[q >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[q] << (16 * (q & 1));
          else w[q] = reinterpret_cast<const uint32_t*>(p)[q];
        }
      }
    }
  }
  __device__ __forceinline__ void put(float* to) const {  // in 32 bits
    if constexpr (sizeof(T) == 2) {
      const float2 a = Elem<T>::to2(w[0]), b = Elem<T>::to2(w[1]);
      *reinterpret_cast<float4*>(to) = make_float4(a.x, a.y, b.x, b.y);
    } else {
      *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
};

__device__ __forceinline__ float2 from_lane(float2 v, int lane) {
  return make_float2(__shfl_sync(0xffffffffu, v.x, lane), __shfl_sync(0xffffffffu, v.y, lane));
}

// Of `tokens` (a multiple of P) tokens' sums over states, a thread's share in each: the whole
// sums of its own tokens, pl, pl + P, .., in v[0], v[P], ..
template <int tokens, int P>
__device__ __forceinline__ void share_out(float2 (&v)[tokens], int pl) {
#pragma unroll
  for (int o = P / 2; o > 0; o >>= 1) {
    const bool up = pl & o;
#pragma unroll
    for (int i = 0; i < tokens; ++i) {
      if (i % P < o) {
        const float2 give = up ? v[i] : v[i + o], keep = up ? v[i + o] : v[i];
        v[i] = add2(keep, make_float2(__shfl_xor_sync(0xffffffffu, give.x, o), __shfl_xor_sync(0xffffffffu, give.y, o)));
      }
    }
  }
}

// Sum over the P threads of a pair; every one gets it.
template <int P>
__device__ __forceinline__ float2 sum_pair(float2 v) {
#pragma unroll
  for (int o = 1; o < P; o <<= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  return v;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

constexpr int64_t kMost = int64_t(1) << 28;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

inline snn_status_t check_desc(const snn_sscan_desc* d) {
  if (!d || d->reserved[0] || d->reserved[1]) return SNN_ERR_INVALID_ARG;
  if (d->B < 0 || d->T < 0 || d->D < 1 || d->N < 1 || d->G < 1 || d->D % d->G) return SNN_ERR_INVALID_ARG;
  if (d->dtype < SNN_F32 || d->dtype > SNN_F16) return SNN_ERR_INVALID_ARG;
  if (d->softplus != 0 && d->softplus != 1) return SNN_ERR_INVALID_ARG;
  if (d->N > kMaxN) return SNN_ERR_UNSUPPORTED;
  // token, channel and block indexes are 32-bit
  if (d->T > kMost || d->B > kMost || d->D > (kMost >> 6) || (d->T > 0 && d->B * d->T > kMost) ||
      d->B * d->D > kMost)
    return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

// A [B, T, D] tensor; *pair is cleared where channel pairs may lie between
// boundaries.
inline snn_status_t take(const snn_sscan_desc* d, const snn_btc* x, Seq* out, bool* pair) {
  if (!x || !x->data) return SNN_ERR_INVALID_ARG;
  if (!aligned16(x->data)) return SNN_ERR_ALIGNMENT;
  const int64_t ext[2] = {d->B, d->T}, str[2] = {x->stride_b, x->stride_t};
  for (int i = 0; i < 2; ++i) {
    if (ext[i] <= 1) continue;
    if (str[i] <= 0 || str[i] >= (int64_t(1) << 38)) return SNN_ERR_INVALID_ARG;
    if (str[i] % 2) *pair = false;
  }
  out->data = x->data;
  out->sb = d->B > 1 ? x->stride_b : 0;
  out->st = d->T > 1 ? x->stride_t : 0;
  return SNN_OK;
}
inline snn_status_t take(const snn_sscan_desc* d, const snn_bthd* x, Mat* out) {
  if (!x || !x->data) return SNN_ERR_INVALID_ARG;
  if (!aligned16(x->data)) return SNN_ERR_ALIGNMENT;
  const int64_t ext[3] = {d->B, d->T, d->G}, str[3] = {x->stride_b, x->stride_t, x->stride_h};
  for (int i = 0; i < 3; ++i)
    if (ext[i] > 1 && (str[i] <= 0 || str[i] >= (int64_t(1) << 38))) return SNN_ERR_INVALID_ARG;
  out->data = x->data;
  out->sb = d->B > 1 ? x->stride_b : 0;
  out->st = d->T > 1 ? x->stride_t : 0;
  out->sg = d->G > 1 ? x->stride_h : 0;
  return SNN_OK;
}

inline bool quads(const Args& g, std::initializer_list<const Mat*> ms) {
  if (g.N % 4) return false;
  for (const Mat* m : ms)
    if ((m->sb | m->st | m->sg) % 4) return false;
  return true;
}

inline Args base_args(const snn_sscan_desc* d) {
  Args g = {};
  g.B = (int)d->B;
  g.T = (int)d->T;
  g.D = (int)d->D;
  g.N = (int)d->N;
  g.G = (int)d->G;
  g.Dg = (int)(d->D / d->G);
  g.softplus = d->softplus;
  g.N2 = (g.N + 1) / 2;
  g.pairs = (g.Dg + 1) / 2;
  return g;
}

// How the axis is cut, from the shape alone.
struct Plan {
  int spans, span, fine, span_fine;
};
// What the kernels of a call need beside its tensors.
inline int64_t state_floats(const Args& g) { return (int64_t)g.B * g.G * g.N2 * g.pairs * 4; }
inline size_t ends_bytes(const Args& g, int spans) { return round256((size_t)(spans * state_floats(g)) * sizeof(float)); }
inline size_t sums_bytes(const Args& g, int spans) {
  return round256((size_t)spans * g.B * g.G * g.pairs * sizeof(float2));
}

}  // namespace sscan
}  // namespace snn
