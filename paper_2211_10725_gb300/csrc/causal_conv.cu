// Causal convolution of each channel over W = 2, 3 or 4 tokens (depthwise), with
// its bias and activation:
//   p_t = bias + sum_j w[j] x_{t-W+1+j},   y_t = act(p_t)
// the inputs before the sequence from a state of W - 1 of them, and its gradients:
//   d_t = grad_y_t act'(p_t);   grad_x_t = sum_j w[j] d_{t+W-1-j}
//   grad_w[j] = sum_t d_t x_{t-W+1+j};   grad_bias = sum_t d_t
// Each tensor is read and written once and a channel-token takes 2 W operations
// beside its activation, so the bound is HBM.  A thread takes four neighbouring channels
// (one vector access) over a run of tokens and keeps the last W - 1 inputs (the
// backward: and gradients) in registers; four tokens' loads are started before the first
// is used.  Neighbouring runs read W - 1 tokens twice, out of L2.  The parameters'
// gradients gather in registers over a run, in shared memory over the runs of a
// block, and a second kernel adds the blocks in their order (no atomics).
//
// 2 x 4096 tokens of 4096 channels, width 4, silu, bf16: forward 30 us (4.5 TB/s), backward
// 57 (3.5) and 6 for the sums; issue at 0.48 and 0.49 a clock, the rest the latency of the loads at 20 and 14 warps
// an SM (one channel's runs of 16 tokens first: 242 us for the three; channels in pairs,
// longer runs: 156; whole fours of tokens without checks: 92; the state read before the tokens: 91).  Eight channels a thread, two or eight tokens ahead
// and other block counts were no faster.  4095 channels, element by element: 163 for 92.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "launch.cuh"
#include "scan_host.cuh"
#include "snn.h"
#include "snn_device.cuh"

namespace snn {
namespace cconv {

constexpr int kThreads = 256;
constexpr int kAhead = 4;      // tokens whose loads are in flight
constexpr int kMinRun = 4;     // at least W - 1: later runs never look at the state
constexpr int kV = 4;          // channels of a thread

struct Tensor {
  void* data = nullptr;
  int64_t sb = 0, st = 0;
};

struct Args {
  Tensor x, y, gy, gx;
  const float *w, *bias;
  const int32_t *seq_lens, *slots;
  const void* state_in;
  void* state_out;
  const void* grad_state_out;
  void* grad_state_in;
  int64_t num_slots;
  int B, T, C, run, runs;
  int silu;
  int step;       // an empty place of the batch writes zeros
  float* part;    // backward: [blocks of runs][C W, then C]
  int lanes;      // backward: threads across the channels
};

// A thread's channels in pairs, one instruction for both (or a single one).
template <int V>
using Lane = typename std::conditional<V == 1, float, float2>::type;
template <int V>
constexpr int kLanes = V == 1 ? 1 : V / 2;
__device__ __forceinline__ float fma2(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float mul2(float a, float b) { return a * b; }
__device__ __forceinline__ float add2(float a, float b) { return a + b; }
using snn::add2;
using snn::fma2;
using snn::mul2;
template <typename L>
__device__ __forceinline__ L all(float a);
template <>
__device__ __forceinline__ float all<float>(float a) { return a; }
template <>
__device__ __forceinline__ float2 all<float2>(float a) { return make_float2(a, a); }
__device__ __forceinline__ float at(float v, int) { return v; }
__device__ __forceinline__ float at(float2 v, int i) { return i ? v.y : v.x; }

// 1 / (1 + e^-p).  Results rounded to 16 bits take the approximate power of
// two and reciprocal: the rounding of p log2(e) costs |p| 2^-24 of the result.
template <typename T>
__device__ __forceinline__ float sigmoid(float p) {
  if constexpr (sizeof(T) == 4) return __frcp_rn(1.0f + expf(-p));
  float e = p * -1.44269504088896340736f;
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e));
  e += 1.0f;
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e));
  return e;
}
template <typename T>
__device__ __forceinline__ float2 sigmoid(float2 p) {
  if constexpr (sizeof(T) == 4) return make_float2(sigmoid<T>(p.x), sigmoid<T>(p.y));
  float2 e = mul2(p, make_float2(-1.44269504088896340736f, -1.44269504088896340736f));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
  e = add2(e, make_float2(1.0f, 1.0f));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e.x));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e.y));
  return e;
}

// V channels as they lie in memory; V = 1 at any element's address.
template <typename T, int V>
struct Vec {
  using L = Lane<V>;
  static constexpr int kWords = V == 1 ? 1 : V * (int)sizeof(T) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (V == 1) {
      if constexpr (sizeof(T) == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
      else w[0] = *reinterpret_cast<const uint16_t*>(p);
    } else if constexpr (kWords == 4) {
      const uint4 a = *reinterpret_cast<const uint4*>(p);
      w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    } else {
      static_assert(kWords == 2, "8 or 16 bytes");
      const uint2 a = *reinterpret_cast<const uint2*>(p);
      w[0] = a.x, w[1] = a.y;
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (V == 1) {
      if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
      else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    } else if constexpr (kWords == 4) {
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
  __device__ __forceinline__ void get(L (&v)[kLanes<V>]) const {
    if constexpr (V == 1) {
      v[0] = Elem<T>::load1(reinterpret_cast<const T*>(w));
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) v[i] = Elem<T>::to2(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) v[i] = make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    }
  }
  __device__ __forceinline__ static void put(T* p, const L (&v)[kLanes<V>]) {
    if constexpr (V == 1) {
      Elem<T>::store1(p, v[0]);
    } else {
      const float a[4] = {v[0].x, v[0].y, v[1].x, v[1].y};
      Elem<T>::store4(p, a);
    }
  }
};

__device__ __forceinline__ int seq_len(const Args& g, int b) {
  if (!g.seq_lens) return g.T;
  const int n = g.seq_lens[b];
  return n < 0 ? 0 : (n > g.T ? g.T : n);
}

// A run of a sequence and this thread's first channel.
template <typename T, int V, int W>
struct Run {
  const Args& g;
  int b, c, len;
  int64_t place;

  __device__ __forceinline__ bool has_place() const { return place >= 0 && place < g.num_slots; }
  __device__ __forceinline__ const T* row(const Tensor& m, int t) const {
    return static_cast<const T*>(m.data) + b * m.sb + t * m.st + c;
  }
  __device__ __forceinline__ T* row_out(const Tensor& m, int t) const {
    return static_cast<T*>(m.data) + b * m.sb + t * m.st + c;
  }
  __device__ __forceinline__ int64_t state_at(int64_t p, int j) const { return (p * (W - 1) + j) * g.C + c; }
  // x_t, from the state before the sequence; zero where there is none
  __device__ __forceinline__ void input(int t, Vec<T, V>& v) const {
    if (t >= 0 && t < len) v.load(row(g.x, t));
    else if (t < 0 && g.state_in && has_place()) v.load(static_cast<const T*>(g.state_in) + state_at(place, W - 1 + t));
    else v.clear();
  }
};

template <int V, int W>
__device__ __forceinline__ void load_params(const Args& g, int c, Lane<V> (&w)[W][kLanes<V>], Lane<V> (&bias)[kLanes<V>]) {
  const float* p = g.w + (int64_t)c * W;  // a thread's channels' taps lie together
  if constexpr (V == 1) {
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][0] = p[j];
    bias[0] = g.bias ? g.bias[c] : 0.0f;
  } else {
    float flat[V * W], b[V] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < V * W; i += 4) Elem<float>::load4(p + i, flat + i);
    if (g.bias) Elem<float>::load4(g.bias + c, b);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
#pragma unroll
      for (int j = 0; j < W; ++j) w[j][i] = make_float2(flat[2 * i * W + j], flat[(2 * i + 1) * W + j]);
      bias[i] = make_float2(b[2 * i], b[2 * i + 1]);
    }
  }
}

template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 2 : 3) conv_fwd(const Args g) {
  constexpr int N = kLanes<V>;
  using L = Lane<V>;
  grid_dep_wait();
  const unsigned cv = g.C / V, unit = blockIdx.x * kThreads + threadIdx.x, lane = unit / cv;
  if (lane >= (unsigned)(g.B * g.runs)) return;
  const int b = (int)(lane / g.runs), r = (int)(lane - b * g.runs);
  const Run<T, V, W> at{g, b, (int)(unit - lane * cv) * V, seq_len(g, b), g.slots ? (int64_t)g.slots[b] : (int64_t)b};
  const int t0 = r * g.run, t1 = t0 + g.run < g.T ? t0 + g.run : g.T;
  const int len = g.step && !at.has_place() ? 0 : at.len;
  L win[W][N];  // x of the last W tokens
  {
    Vec<T, V> first[W - 1];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      first[j].clear();
      if (t0 < len) at.input(t0 - (W - 1) + j, first[j]);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) first[j].get(win[j + 1]);
  }
  L w[W][N], bias[N];
  load_params<V, W>(g, at.c, w, bias);
  const T* px = at.row(g.x, t0);
  T* py = at.row_out(g.y, t0);
  Vec<T, V> raw[kAhead];
  const int stop = t1 < len ? t1 : len;
  auto fetch = [&](int t) {
    if (t + kAhead <= stop) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) raw[i].load(px + i * g.x.st);
    } else {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        raw[i].clear();
        if (t + i < stop) raw[i].load(px + i * g.x.st);
      }
    }
    px += kAhead * g.x.st;
  };
  // whole: all the tokens exist
  auto tokens = [&](int t, auto whole) {
    Vec<T, V> now[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) now[i] = raw[i];
    fetch(t + kAhead);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (decltype(whole)::value || t + i < t1) {
        L y[N];
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
          for (int v = 0; v < N; ++v) win[j][v] = win[j + 1][v];
        now[i].get(win[W - 1]);
#pragma unroll
        for (int v = 0; v < N; ++v) {
          L p = bias[v];
#pragma unroll
          for (int j = 0; j < W; ++j) p = fma2(w[j][v], win[j][v], p);
          if (g.silu) p = mul2(p, sigmoid<T>(p));
          y[v] = decltype(whole)::value || t + i < len ? p : all<L>(0.0f);
        }
        Vec<T, V>::put(py + i * g.y.st, y);
      }
    }
    py += kAhead * g.y.st;
  };
  fetch(t0);
  // the last W - 1 inputs; in ascending order, as state_out may be state_in, and before y,
  // which a step's x may be
  if (r == 0 && g.state_out && at.has_place()) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      Vec<T, V> v;
      at.input(at.len - (W - 1) + j, v);
      v.store(static_cast<T*>(g.state_out) + at.state_at(at.place, j));
    }
  }
  int t = t0;
  for (; t + kAhead <= stop; t += kAhead) tokens(t, std::true_type());
  for (; t < t1; t += kAhead) tokens(t, std::false_type());
}

template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 1 : 2) conv_bwd(const Args g) {
  extern __shared__ float conv_smem[];  // [runs of a block][lanes V][W + 1]
  constexpr int N = kLanes<V>;
  using L = Lane<V>;
  grid_dep_wait();
  const int lanes = g.lanes, rows = kThreads / lanes, cv = g.C / V;
  const int cblocks = (cv + lanes - 1) / lanes, rblocks = (g.runs + rows - 1) / rows;
  const int cb = (int)(blockIdx.x % (unsigned)cblocks), rest = (int)(blockIdx.x / (unsigned)cblocks);
  const int rb = rest % rblocks, b = rest / rblocks;
  const int lane = threadIdx.x % lanes, ty = threadIdx.x / lanes;
  const int vec = cb * lanes + lane, r = rb * rows + ty;
  const L zero = all<L>(0.0f);
  L dw[W][N], db[N];
#pragma unroll
  for (int v = 0; v < N; ++v) {
    db[v] = zero;
#pragma unroll
    for (int j = 0; j < W; ++j) dw[j][v] = zero;
  }
  if (vec < cv && r < g.runs) {
    const Run<T, V, W> at{g, b, vec * V, seq_len(g, b), (int64_t)b};
    const int t0 = r * g.run, t1 = t0 + g.run < g.T ? t0 + g.run : g.T, len = at.len;
    const int end = t1 + W - 1;  // token t gives grad_x of token t - W + 1
    L w[W][N], bias[N], win[W][N], d[W][N];  // the last W inputs; the last W gradients
    load_params<V, W>(g, at.c, w, bias);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      Vec<T, V> first;
      first.clear();
      if (t0 < len) at.input(t0 - (W - 1) + j, first);
      first.get(win[j + 1]);
    }
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int v = 0; v < N; ++v) d[j][v] = zero;
    const T *px = at.row(g.x, t0), *pg = at.row(g.gy, t0);
    T* po = at.row_out(g.gx, t0) - (W - 1) * g.gx.st;
    Vec<T, V> raw[kAhead], raw_gy[kAhead];
    const int stop = end < len ? end : len;
    auto fetch = [&](int t) {
      if (t + kAhead <= stop) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          raw[i].load(px + i * g.x.st);
          raw_gy[i].load(pg + i * g.gy.st);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          raw[i].clear();
          raw_gy[i].clear();
          if (t + i < stop) {
            raw[i].load(px + i * g.x.st);
            raw_gy[i].load(pg + i * g.gy.st);
          }
        }
      }
      px += kAhead * g.x.st;
      pg += kAhead * g.gy.st;
    };
    // whole: all the tokens exist and are the run's own, as are those W - 1 before them
    auto tokens = [&](int t, auto whole_) {
      constexpr bool whole = decltype(whole_)::value;
      Vec<T, V> now_x[kAhead], now_gy[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) now_x[i] = raw[i], now_gy[i] = raw_gy[i];
      fetch(t + kAhead);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int now = t + i;
        if (whole || now < end) {
          L gx[N], gy[N];
#pragma unroll
          for (int j = 0; j < W - 1; ++j)
#pragma unroll
            for (int v = 0; v < N; ++v) win[j][v] = win[j + 1][v], d[j][v] = d[j + 1][v];
          now_x[i].get(win[W - 1]);
          now_gy[i].get(gy);
#pragma unroll
          for (int v = 0; v < N; ++v) {
            L dt = gy[v];
            if (g.silu) {
              L p = bias[v];
#pragma unroll
              for (int j = 0; j < W; ++j) p = fma2(w[j][v], win[j][v], p);
              const L s = sigmoid<T>(p);
              dt = mul2(dt, fma2(mul2(p, s), fma2(s, all<L>(-1.0f), all<L>(1.0f)), s));
            }
            if (!whole && now >= len) dt = zero;
            d[W - 1][v] = dt;
            if (whole || (now < t1 && now < len)) {
              db[v] = add2(db[v], dt);
#pragma unroll
              for (int j = 0; j < W; ++j) dw[j][v] = fma2(dt, win[j][v], dw[j][v]);
            }
            gx[v] = mul2(w[0][v], d[W - 1][v]);
#pragma unroll
            for (int j = 1; j < W; ++j) gx[v] = fma2(w[j][v], d[W - 1 - j][v], gx[v]);
          }
          const int to = now - (W - 1);
          if (whole) {
            if (g.gx.data) Vec<T, V>::put(po + i * g.gx.st, gx);
          } else if (to >= t0 || r == 0) {
            const int j = to - (len - (W - 1));  // the row of the last inputs that this one is
            if (g.grad_state_out && j >= 0 && j < W - 1) {
              Vec<T, V> s;
              s.load(static_cast<const T*>(g.grad_state_out) + at.state_at(b, j));
              s.get(gy);
#pragma unroll
              for (int v = 0; v < N; ++v) gx[v] = add2(gx[v], gy[v]);
            }
            if (to >= len)
#pragma unroll
              for (int v = 0; v < N; ++v) gx[v] = zero;
            if (to >= 0) {
              if (g.gx.data) Vec<T, V>::put(po + i * g.gx.st, gx);
            } else if (g.grad_state_in) {
              Vec<T, V>::put(static_cast<T*>(g.grad_state_in) + at.state_at(b, W - 1 + to), gx);
            }
          }
        }
      }
      po += kAhead * g.gx.st;
    };
    fetch(t0);
    int t = t0;
    for (; t < end && t < t0 + W - 1; t += kAhead) tokens(t, std::false_type());
    for (; t + kAhead <= t1 && t + kAhead <= len; t += kAhead) tokens(t, std::true_type());
    for (; t < end; t += kAhead) tokens(t, std::false_type());
  }
  if (!g.part) return;
  const int width = lanes * V;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float* s = conv_smem + ((int64_t)ty * width + lane * V + v) * (W + 1);
#pragma unroll
    for (int j = 0; j < W; ++j) s[j] = cconv::at(dw[j][v / 2], v & 1);
    s[W] = cconv::at(db[v / 2], v & 1);
  }
  __syncthreads();
  float* part = g.part + (int64_t)rest * g.C * (W + 1);
  for (int i = threadIdx.x; i < width * (W + 1); i += kThreads) {
    const int ch = i / (W + 1), j = i - ch * (W + 1), c = cb * width + ch;
    if (c >= g.C) continue;
    float v = conv_smem[i];
    for (int k = 1; k < rows; ++k) v += conv_smem[(int64_t)k * width * (W + 1) + i];
    part[j < W ? (int64_t)c * W + j : (int64_t)g.C * W + c] = v;
  }
}

// Column sums of the partials: 32 columns a block, the rows in 32 slices (every
// 32nd row, in order), then the slices in order.
__global__ void __launch_bounds__(1024) conv_sum(const float* __restrict__ part, int64_t rows, int64_t width,
                                                 int64_t split, float* grad_w, float* grad_b) {
  __shared__ float s[32][33];
  grid_dep_wait();
  const int64_t c = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
  const int slice = threadIdx.x >> 5;
  float v = 0.0f;
  if (c < width) {
#pragma unroll 4
    for (int64_t i = slice; i < rows; i += 32) v += part[i * width + c];
  }
  s[slice][threadIdx.x & 31] = v;
  __syncthreads();
  if (slice || c >= width) return;
  for (int i = 1; i < 32; ++i) v += s[i][threadIdx.x];
  if (c < split) {
    if (grad_w) grad_w[c] = v;
  } else if (grad_b) {
    grad_b[c - split] = v;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

constexpr int64_t kMost = int64_t(1) << 28;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

snn_status_t check_desc(const snn_conv_desc* d) {
  if (!d || d->reserved[0] || d->reserved[1]) return SNN_ERR_INVALID_ARG;
  if (d->B < 0 || d->T < 0 || d->C < 1 || d->W < 1) return SNN_ERR_INVALID_ARG;
  if (d->dtype < SNN_F32 || d->dtype > SNN_F16) return SNN_ERR_INVALID_ARG;
  if (d->act != SNN_GATE_NONE && d->act != SNN_GATE_SILU)
    return d->act == SNN_GATE_SIGMOID ? SNN_ERR_UNSUPPORTED : SNN_ERR_INVALID_ARG;
  if (d->W < 2 || d->W > 4) return SNN_ERR_UNSUPPORTED;
  // token, channel and block indexes are 32-bit
  if (d->T > kMost || d->B > kMost || d->C > kMost || (d->B > 0 && d->T > 0 && d->B * d->T > kMost))
    return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

// A [B, T, C] tensor; *vec is cleared where its rows are not whole vectors apart.
snn_status_t take(const snn_conv_desc* d, const snn_btc* x, Tensor* out, bool* vec) {
  if (!x || !x->data) return SNN_ERR_INVALID_ARG;
  if (!aligned16(x->data)) return SNN_ERR_ALIGNMENT;
  const int64_t ext[2] = {d->B, d->T}, str[2] = {x->stride_b, x->stride_t};
  for (int i = 0; i < 2; ++i) {
    if (ext[i] <= 1) continue;
    if (str[i] <= 0 || str[i] >= (int64_t(1) << 38)) return SNN_ERR_INVALID_ARG;
    if (str[i] % kV) *vec = false;
  }
  out->data = x->data;
  out->sb = d->B > 1 ? x->stride_b : 0;
  out->st = d->T > 1 ? x->stride_t : 0;
  return SNN_OK;
}

int lanes_for(int64_t vecs) { return vecs <= 8 ? 8 : vecs <= 16 ? 16 : 32; }

// Tokens of a run: few enough to fill the GPU with threads, at most `most` (the
// tokens that two runs share and a run's partial sums cost less in longer ones).
// Threads that fill an SM: forward 1536 (6 x 1500 tokens of 2056 channels: 14.9 us, 17.4 with 768),
// backward, which has fewer registers and sums to hand on, 768 (forward and backward of
// 2 x 4096 tokens of 4096 channels: 92.3 us, 98.7 with 1536).
constexpr int64_t kFwdFill = 152 * 1536, kBwdFill = 152 * 768;
int run_length(int64_t B, int64_t T, int64_t threads_across, int most, int64_t fill) {
  int run = most;
  while (run > kMinRun && B * snn::ceil_div(T, run) * threads_across < fill) run /= 2;
  return run;
}

// The backward's plan, from the shape alone (the vectors of the odd path are
// elements; its runs are the same, so that the workspace does not depend on strides).
struct BwdPlan {
  int run, runs;
};
BwdPlan bwd_plan(int64_t B, int64_t T, int64_t C) {
  BwdPlan p;
  p.run = run_length(B, T, snn::ceil_div(C, kV), 64, kBwdFill);
  p.runs = T > 0 ? (int)snn::ceil_div(T, p.run) : 1;  // of no tokens: the states' gradients pass through
  return p;
}
int64_t bwd_rows(const BwdPlan& p, int64_t B, int64_t vecs) { return B * snn::ceil_div(p.runs, kThreads / lanes_for(vecs)); }

template <typename T, int V, int W>
cudaError_t launch_fwd(Args g, cudaStream_t st) {
  g.run = run_length(g.B, g.T, g.C / V, 32, kFwdFill);
  g.runs = g.T > 0 ? (int)snn::ceil_div(g.T, g.run) : 1;  // of no tokens: the states pass through
  const int64_t units = (int64_t)g.B * g.runs * (g.C / V), blocks = snn::ceil_div(units, kThreads);
  if (units > 0x7fffff00) return cudaErrorInvalidValue;
  return launch_pdl(conv_fwd<T, V, W>, dim3((unsigned)blocks), dim3(kThreads), 0, st, g);
}

template <typename T, int V, int W>
cudaError_t launch_bwd(Args g, cudaStream_t st) {
  const int64_t vecs = g.C / V;
  g.lanes = lanes_for(vecs);
  const BwdPlan p = bwd_plan(g.B, g.T, g.C);
  g.run = p.run;
  g.runs = p.runs;
  const int64_t blocks = bwd_rows(p, g.B, vecs) * snn::ceil_div(vecs, g.lanes);
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  const size_t smem = (size_t)kThreads * V * (W + 1) * sizeof(float);
  return launch_pdl(conv_bwd<T, V, W>, dim3((unsigned)blocks), dim3(kThreads), smem, st, g);
}

template <typename T, int W>
cudaError_t launch_width(const Args& g, bool bwd, bool vec, cudaStream_t st) {
  if (bwd) return vec ? launch_bwd<T, kV, W>(g, st) : launch_bwd<T, 1, W>(g, st);
  return vec ? launch_fwd<T, kV, W>(g, st) : launch_fwd<T, 1, W>(g, st);
}

template <typename T>
cudaError_t launch_type(const Args& g, int W, bool bwd, bool vec, cudaStream_t st) {
  if (W == 2) return launch_width<T, 2>(g, bwd, vec, st);
  if (W == 3) return launch_width<T, 3>(g, bwd, vec, st);
  return launch_width<T, 4>(g, bwd, vec, st);
}

cudaError_t launch(const snn_conv_desc* d, const Args& g, bool bwd, bool vec, cudaStream_t st) {
  if (d->dtype == SNN_F32) return launch_type<float>(g, (int)d->W, bwd, vec, st);
  if (d->dtype == SNN_BF16) return launch_type<__nv_bfloat16>(g, (int)d->W, bwd, vec, st);
  return launch_type<__half>(g, (int)d->W, bwd, vec, st);
}

Args base_args(const snn_conv_desc* d, const float* w, const float* bias) {
  Args g = {};
  g.B = (int)d->B;
  g.T = (int)d->T;
  g.C = (int)d->C;
  g.silu = d->act == SNN_GATE_SILU;
  g.w = w;
  g.bias = bias;
  return g;
}

snn_status_t forward(const snn_conv_desc* d, const snn_btc* x, const float* w, const float* bias,
                     const int32_t* seq_lens, const void* state_in, void* state_out, const int32_t* slots,
                     int64_t num_slots, const snn_btc* y, bool step, snn_stream_t stream) {
  const void* ptrs[6] = {w, bias, seq_lens, state_in, state_out, slots};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  if (!w || num_slots < 0 || num_slots > kMost) return SNN_ERR_INVALID_ARG;
  if ((state_in || state_out) && !slots && num_slots < d->B) return SNN_ERR_INVALID_ARG;
  Args g = base_args(d, w, bias);
  bool vec = d->C % kV == 0;
  snn_status_t s;
  if (d->B == 0) return SNN_OK;
  if (d->T > 0 && ((s = take(d, x, &g.x, &vec)) != SNN_OK || (s = take(d, y, &g.y, &vec)) != SNN_OK)) return s;
  if (d->T == 0 && !state_out) return SNN_OK;
  g.seq_lens = seq_lens;
  g.state_in = state_in;
  g.state_out = state_out;
  g.slots = slots;
  g.num_slots = num_slots;
  g.step = step;
  return launch(d, g, false, vec, reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

}  // namespace cconv
}  // namespace snn

using namespace snn::cconv;

extern "C" {

size_t snn_conv_desc_size(void) { return sizeof(snn_conv_desc); }

size_t snn_causal_conv_workspace_bytes(const snn_conv_desc* desc) {
  if (check_desc(desc) != SNN_OK) return 0;
  // rows of partials of the element path and of the vector path: the larger
  const BwdPlan p = bwd_plan(desc->B, desc->T, desc->C);
  const int64_t a = bwd_rows(p, desc->B, desc->C), v = bwd_rows(p, desc->B, snn::ceil_div(desc->C, kV));
  const size_t b = (size_t)(a > v ? a : v) * (size_t)desc->C * (size_t)(desc->W + 1) * sizeof(float);
  return b < 256 ? 256 : b;
}

snn_status_t snn_causal_conv_fwd(const snn_conv_desc* desc, const snn_btc* x, const float* w,
                                 const float* bias, const int32_t* seq_lens, const void* state_in,
                                 void* state_out, const int32_t* slots, int64_t num_slots,
                                 const snn_btc* y, snn_stream_t stream) {
  const snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  return forward(desc, x, w, bias, seq_lens, state_in, state_out, slots, num_slots, y, false, stream);
}

snn_status_t snn_causal_conv_step(const snn_conv_desc* desc, const snn_btc* x, const float* w,
                                  const float* bias, void* state, const int32_t* slots,
                                  int64_t num_slots, const snn_btc* y, snn_stream_t stream) {
  const snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  if (desc->T != 1 || !state) return SNN_ERR_INVALID_ARG;
  return forward(desc, x, w, bias, nullptr, state, state, slots, num_slots, y, true, stream);
}

snn_status_t snn_causal_conv_bwd(const snn_conv_desc* desc, const snn_btc* x, const float* w,
                                 const float* bias, const int32_t* seq_lens, const void* state_in,
                                 const snn_btc* grad_y, const void* grad_state_out, const snn_btc* grad_x,
                                 float* grad_w, float* grad_bias, void* grad_state_in, void* ws,
                                 size_t ws_bytes, snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  const void* ptrs[9] = {w, bias, seq_lens, state_in, grad_state_out, grad_w, grad_bias, grad_state_in, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  if (!w) return SNN_ERR_INVALID_ARG;
  if (grad_state_in && (grad_state_in == state_in || grad_state_in == grad_state_out)) return SNN_ERR_INVALID_ARG;
  const bool params = grad_w || grad_bias;
  if (params && (!ws || ws_bytes < snn_causal_conv_workspace_bytes(desc))) return SNN_ERR_WORKSPACE;
  Args g = base_args(desc, w, bias);
  bool vec = desc->C % kV == 0;
  if (desc->B > 0 && desc->T > 0) {
    if ((s = take(desc, x, &g.x, &vec)) != SNN_OK || (s = take(desc, grad_y, &g.gy, &vec)) != SNN_OK ||
        (grad_x && grad_x->data && (s = take(desc, grad_x, &g.gx, &vec)) != SNN_OK))
      return s;
  }
  g.seq_lens = seq_lens;
  g.state_in = state_in;
  g.grad_state_out = grad_state_out;
  g.grad_state_in = grad_state_in;
  g.num_slots = desc->B;
  g.part = params ? static_cast<float*>(ws) : nullptr;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const BwdPlan p = bwd_plan(desc->B, desc->T, desc->C);
  const int64_t rows = bwd_rows(p, desc->B, vec ? desc->C / kV : desc->C);
  cudaError_t e = cudaSuccess;
  if (rows > 0 && (params || g.gx.data || grad_state_in)) e = launch(desc, g, true, vec, st);
  if (e == cudaSuccess && params) {
    const int64_t width = desc->C * (desc->W + 1);
    e = snn::launch_pdl(conv_sum, dim3((unsigned)snn::ceil_div(width, 32)), dim3(1024), 0, st,
                        static_cast<const float*>(ws), rows, width, desc->C * desc->W, grad_w, grad_bias);
  }
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

}  // extern "C"
