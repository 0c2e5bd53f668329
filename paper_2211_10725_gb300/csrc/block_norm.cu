// Block norms: the norm after a block, its gate and residual scale, the
// residual sum and the norm before the next block, per row of N channels:
//   n  = a rstd_a w_post            rstd_a = rsqrt(mean over the group of a^2 + eps)
//   r' = r + s n act(z)
//   y  = r' rstd w_pre              rstd   = rsqrt(mean over the row of r'^2 + eps)
// and the gradients (g = grad_y w_pre, e = r' rstd):
//   d      = grad_r' + rstd (g - e mean(g e))
//   grad_r = d;  grad_z = d s n act'(z)
//   grad_a = rstd_a (m - h mean_group(m h)),  h = a rstd_a,  m = d s act(z) w_post
//   grad_w_post = s G,  grad_s = w_post G  with  G = sum d act(z) h;  grad_w_pre = sum grad_y e
// Every tensor is read and written once: the bound is HBM.  A row stays in
// the registers of one warp (short rows) or one block, eight channels to a
// thread; blocks stay on the GPU and take rows in turn, with the next row's
// loads in flight while the sums of the present one meet.  The parameters'
// gradients gather in the registers (long rows: in shared memory) of the
// thread that owns the channels over all the rows of its block, so the sums
// over rows need one [blocks, 2, N] array of partials and a second kernel
// that adds them in block order (no atomics: the same bits on every call).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "launch.cuh"
#include "scan_host.cuh"
#include "snn.h"
#include "snn_device.cuh"

namespace snn {
namespace norm {

constexpr int64_t kMaxN = 8192;
constexpr int kSms = 152;
constexpr int E = 8;  // channels of a thread

struct Rows {
  void* data;
  int64_t ld;
};

struct Args {
  int64_t M;
  int N, group, gate;
  float eps;
  Rows r, a, z, ro, y;        // forward
  Rows gro, gy, gr, ga, gz;   // backward (reads ro, a, z)
  const float *w_post, *scale, *w_pre;
  float* part;                // [blocks][2][N]
};

__device__ __forceinline__ float sigmoidf_(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }

// Eight floats as one 32-byte access (p 32-byte aligned): two 16-byte ones
// would each touch half of every 32-byte sector.
__device__ __forceinline__ void load32(const float* p, uint4 w[2]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0].x), "=r"(w[0].y), "=r"(w[0].z), "=r"(w[0].w), "=r"(w[1].x), "=r"(w[1].y),
                 "=r"(w[1].z), "=r"(w[1].w)
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store32(float* p, const float v[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]),
               "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}

// A thread's share of a row as it lies in memory: eight consecutive channels
// (VEC), else every TPR-th.
template <typename T, bool VEC, int TPR>
struct Share {
  static constexpr int kWords = E * sizeof(T) / 16;
  uint4 w[VEC ? kWords : 1];
  T x[VEC ? 1 : E];

  __device__ __forceinline__ void load(const Rows& m, int64_t row, int N, int t) {
    const T* p = static_cast<const T*>(m.data) + row * m.ld;
    if constexpr (VEC) {
      if (t * E < N) {
        if constexpr (sizeof(T) == 4) load32(reinterpret_cast<const float*>(p + t * E), w);
        else
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const uint4*>(p + t * E)[i];
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e * TPR + t < N) x[e] = p[e * TPR + t];
    }
  }
  // in 32 bits, zero past N
  __device__ __forceinline__ void get(int N, int t, float v[E]) const {
    if constexpr (VEC) {
      if (t * E < N) {
        Elem<T>::load8(reinterpret_cast<const T*>(w), v);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = 0.0f;
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = e * TPR + t < N ? (float)x[e] : 0.0f;
    }
  }
};

template <typename T, bool VEC, int TPR>
__device__ __forceinline__ void store_row(const Rows& m, int64_t row, int N, int t, const float v[E]) {
  T* p = static_cast<T*>(m.data) + row * m.ld;
  if constexpr (VEC) {
    if (t * E < N) {
      if constexpr (sizeof(T) == 4) store32(p + t * E, v);
      else Elem<T>::store8(p + t * E, v);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e * TPR + t < N) Elem<T>::store1(p + e * TPR + t, v[e]);
  }
}

// A parameter's share (ones where it is absent, zero past N).
template <bool VEC, int TPR>
__device__ __forceinline__ void load_param(const float* p, int N, int t, float v[E]) {
  if (VEC && p && t * E < N) {
    Elem<float>::load8(p + t * E, v);
    return;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int c = VEC ? t * E + e : e * TPR + t;
    v[e] = c < N ? (p ? p[c] : 1.0f) : 0.0f;
  }
}

// Sums of K values over the TPR threads of a row; every thread gets them.
// Successive sums alternate between two scratch buffers, so one barrier a sum
// is enough: a warp cannot be two sums ahead.
template <int TPR>
struct RowSum {
  float (*scratch)[3][32];  // [2][value][warp]
  int turn = 0;
  template <int K>
  __device__ __forceinline__ void operator()(float (&v)[K]) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    if constexpr (TPR > 32) {
      constexpr int W = TPR / 32;
      float (*s)[32] = scratch[turn];
      turn ^= 1;
      if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) s[k][threadIdx.x >> 5] = v[k];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) {
        float a = 0.0f;
#pragma unroll
        for (int w = 0; w < W; w += 4) {
          const float4 x = *reinterpret_cast<const float4*>(&s[k][w]);
          a += (x.x + x.y) + (x.z + x.w);
        }
        v[k] = a;
      }
    }
  }
};

// Sum over the group of `lanes` neighbouring threads that a vector lies in.
__device__ __forceinline__ float group_sum(float v, int lanes) {
  for (int o = 1; o < lanes; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <int TPR>
constexpr int kBlockThreads = TPR == 32 ? 256 : TPR;  // short rows: eight warps, a row each

// Registers: two blocks of 512 threads (or as many smaller ones) on an SM,
// one of 1024.
template <typename T, typename R, bool VEC, int TPR>
__global__ void __launch_bounds__(kBlockThreads<TPR>, 1024 / kBlockThreads<TPR>) norm_fwd(const Args g) {
  __shared__ __align__(16) float scratch[2][3][32];
  grid_dep_wait();
  constexpr int kTeams = kBlockThreads<TPR> / TPR;
  const int t = threadIdx.x % TPR, N = g.N;
  const int64_t step = (int64_t)gridDim.x * kTeams;
  int64_t row = (int64_t)blockIdx.x * kTeams + threadIdx.x / TPR;
  const bool whole = g.group == N, block = g.a.data != nullptr, gated = g.z.data != nullptr;
  const float inv_n = 1.0f / (float)N, inv_g = 1.0f / (float)g.group;
  RowSum<TPR> row_sum{scratch};
  float w_post[E], w_pre[E];
  load_param<VEC, TPR>(g.w_pre, N, t, w_pre);
  if (block) {  // s n act(z): the two factors of a channel as one
    float sc[E];
    load_param<VEC, TPR>(g.w_post, N, t, w_post);
    load_param<VEC, TPR>(g.scale, N, t, sc);
#pragma unroll
    for (int e = 0; e < E; ++e) w_post[e] *= sc[e];
  }
  Share<R, VEC, TPR> r;
  Share<T, VEC, TPR> a, z;
  auto fetch = [&](int64_t i) {
    r.load(g.r, i, N, t);
    if (block) a.load(g.a, i, N, t);
    if (gated) z.load(g.z, i, N, t);
  };
  if (row < g.M) fetch(row);
  for (; row < g.M; row += step) {
    float x[E], u[E], sg[E];
    r.get(N, t, x);
    if (block) a.get(N, t, u);
    if (gated) z.get(N, t, sg);
    if (row + step < g.M) fetch(row + step);
    if (block) {
      float ss[1] = {0.0f};
#pragma unroll
      for (int e = 0; e < E; ++e) ss[0] = fmaf(u[e], u[e], ss[0]);
      if (whole) row_sum(ss);
      else ss[0] = group_sum(ss[0], g.group >> 3);
      const float rstd = rsqrtf(fmaf(ss[0], whole ? inv_n : inv_g, g.eps));
#pragma unroll
      for (int e = 0; e < E; ++e) {
        u[e] = u[e] * rstd * w_post[e];
        if (gated) {
          const float s = sigmoidf_(sg[e]);
          u[e] *= g.gate == SNN_GATE_SILU ? sg[e] * s : s;
        }
        x[e] += u[e];
      }
      store_row<R, VEC, TPR>(g.ro, row, N, t, x);
    }
    if (g.y.data) {
      float ss[1] = {0.0f};
#pragma unroll
      for (int e = 0; e < E; ++e) ss[0] = fmaf(x[e], x[e], ss[0]);
      row_sum(ss);
      const float rstd = rsqrtf(fmaf(ss[0], inv_n, g.eps));
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = x[e] * rstd * w_pre[e];
      store_row<T, VEC, TPR>(g.y, row, N, t, x);
    }
  }
}

// Two vectors of a thread's channels that live as long as its block: in
// registers, or (long rows, whose threads have none to spare) in shared
// memory, [4][E / 4][threads] float4 with the pair at FIRST.
template <bool SMEM, int THREADS, int FIRST>
struct Kept {
  float v[SMEM ? 1 : 2][E];
  __device__ __forceinline__ float4& at(int k, int i) {
    extern __shared__ float4 kept_smem[];
    return kept_smem[((FIRST + k) * (E / 4) + i) * THREADS + threadIdx.x];
  }
  __device__ __forceinline__ void set(int k, const float (&a)[E]) {
    if constexpr (SMEM) {
#pragma unroll
      for (int i = 0; i < E / 4; ++i) at(k, i) = make_float4(a[4 * i], a[4 * i + 1], a[4 * i + 2], a[4 * i + 3]);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = a[e];
    }
  }
  __device__ __forceinline__ void get(int k, float (&a)[E]) {
    if constexpr (SMEM) {
#pragma unroll
      for (int i = 0; i < E / 4; ++i) {
        const float4 s = at(k, i);
        a[4 * i] = s.x;
        a[4 * i + 1] = s.y;
        a[4 * i + 2] = s.z;
        a[4 * i + 3] = s.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) a[e] = v[k][e];
    }
  }
  __device__ __forceinline__ void add(int k, const float (&a)[E], const float (&b)[E]) {  // += a b
    float s[E];
    get(k, s);
#pragma unroll
    for (int e = 0; e < E; ++e) s[e] = fmaf(a[e], b[e], s[e]);
    set(k, s);
  }
};

template <typename T, typename R, bool VEC, int TPR>
__global__ void __launch_bounds__(kBlockThreads<TPR>, TPR == 1024 ? 1 : 512 / kBlockThreads<TPR>)
    norm_bwd(const Args g) {
  __shared__ __align__(16) float scratch[2][3][32];
  grid_dep_wait();
  constexpr int kTeams = kBlockThreads<TPR> / TPR;
  const int t = threadIdx.x % TPR, team = threadIdx.x / TPR, N = g.N;
  const int64_t step = (int64_t)gridDim.x * kTeams;
  int64_t row = (int64_t)blockIdx.x * kTeams + team;
  const bool whole = g.group == N, block = g.a.data != nullptr, gated = g.z.data != nullptr;
  const bool pre = g.gy.data != nullptr, through = g.gro.data != nullptr;
  const float inv_n = 1.0f / (float)N, inv_g = 1.0f / (float)g.group;
  RowSum<TPR> row_sum{scratch};
  // 0: of d act(z) h, 1: of grad_y y';  0: w_pre, 1: s w_post
  Kept<TPR == 1024, TPR, 0> sums;
  Kept<TPR == 1024, TPR, 2> params;
  {
    float w[E], sc[E];
    load_param<VEC, TPR>(g.w_pre, N, t, w);
    params.set(0, w);
    load_param<VEC, TPR>(g.w_post, N, t, w);
    load_param<VEC, TPR>(g.scale, N, t, sc);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      w[e] *= sc[e];
      sc[e] = 0.0f;
    }
    params.set(1, w);
    sums.set(0, sc);
    sums.set(1, sc);
  }
  Share<R, VEC, TPR> ro, gro;
  Share<T, VEC, TPR> gy, a, z;
  auto fetch = [&](int64_t i) {
    if (pre) ro.load(g.ro, i, N, t);
    if (pre) gy.load(g.gy, i, N, t);
    if (through) gro.load(g.gro, i, N, t);
    if (block) a.load(g.a, i, N, t);
    if (gated) z.load(g.z, i, N, t);
  };
  // long rows have not the registers to hold a row ahead
  constexpr bool kAhead = TPR < 1024;
  if (kAhead && row < g.M) fetch(row);
  for (; row < g.M; row += step) {
    if (!kAhead) fetch(row);
    float d[E], x[E], gw[E], h[E], zz[E];
    if (pre) ro.get(N, t, x);
    if (pre) gy.get(N, t, gw);
    if (block) a.get(N, t, h);
    if (gated) z.get(N, t, zz);
    if (through) {
      gro.get(N, t, d);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = 0.0f;
    }
    if (kAhead && row + step < g.M) fetch(row + step);
    float ss[3] = {0.0f, 0.0f, 0.0f};  // of r'^2, grad_y w_pre r', a^2
    float w[E];
    params.get(0, w);
    if (pre) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        ss[0] = fmaf(x[e], x[e], ss[0]);
        ss[1] = fmaf(gw[e] * w[e], x[e], ss[1]);
      }
    }
    if (block) {
#pragma unroll
      for (int e = 0; e < E; ++e) ss[2] = fmaf(h[e], h[e], ss[2]);
    }
    float in_group = 0.0f;
    if (block && !whole) in_group = group_sum(ss[2], g.group >> 3);
    row_sum(ss);
    if (pre) {
      const float rstd = rsqrtf(fmaf(ss[0], inv_n, g.eps));
      const float mean = ss[1] * rstd * inv_n;  // mean of (grad_y w_pre) y'
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] *= rstd;  // y'
      sums.add(1, gw, x);
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = fmaf(rstd, fmaf(-x[e], mean, gw[e] * w[e]), d[e]);
    }
    if (g.gr.data) store_row<R, VEC, TPR>(g.gr, row, N, t, d);
    if (!block) continue;
    const float rstd_a = rsqrtf(whole ? fmaf(ss[2], inv_n, g.eps) : fmaf(in_group, inv_g, g.eps));
    float q[1] = {0.0f};
    params.get(1, w);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      h[e] *= rstd_a;
      x[e] = d[e];
      d[e] *= w[e];
      if (gated) {
        const float s = sigmoidf_(zz[e]);
        const float act = g.gate == SNN_GATE_SILU ? zz[e] * s : s;
        const float slope = g.gate == SNN_GATE_SILU ? s * fmaf(zz[e], 1.0f - s, 1.0f) : s * (1.0f - s);
        zz[e] = d[e] * h[e] * slope;  // grad_z
        x[e] *= act;
        d[e] *= act;                  // m
      }
      q[0] = fmaf(d[e], h[e], q[0]);
    }
    sums.add(0, x, h);
    if (g.gz.data) store_row<T, VEC, TPR>(g.gz, row, N, t, zz);
    if (!g.ga.data) continue;
    if (whole) row_sum(q);
    else q[0] = group_sum(q[0], g.group >> 3);
    const float mean = q[0] * (whole ? inv_n : inv_g);
#pragma unroll
    for (int e = 0; e < E; ++e) d[e] = rstd_a * fmaf(-h[e], mean, d[e]);
    store_row<T, VEC, TPR>(g.ga, row, N, t, d);
  }
  if (!g.part) return;
  float* p = g.part + (int64_t)blockIdx.x * 2 * N;
  if constexpr (kTeams > 1) {  // the block's teams, in order
    __shared__ float all[kTeams][2][TPR * E];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float v[E];
      sums.get(k, v);
#pragma unroll
      for (int e = 0; e < E; ++e) all[team][k][VEC ? t * E + e : e * TPR + t] = v[e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * N; i += kBlockThreads<TPR>) {
      const int k = i / N, at = i - k * N;
      float v = all[0][k][at];
#pragma unroll
      for (int j = 1; j < kTeams; ++j) v += all[j][k][at];
      p[i] = v;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float v[E];
      sums.get(k, v);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int at = VEC ? t * E + e : e * TPR + t;
        if (at < N) p[k * N + at] = v[e];
      }
    }
  }
}

// Column sums of the partials: 32 columns a block, the rows in 32 slices (every
// 32nd row, in order), then the slices in order.
__global__ void __launch_bounds__(1024) norm_sum(const float* __restrict__ part, int rows, int N,
                                                 const float* w_post, const float* scale,
                                                 float* g_post, float* g_scale, float* g_pre) {
  __shared__ float s[32][33];
  grid_dep_wait();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31);
  const int slice = threadIdx.x >> 5, width = 2 * N;
  float v = 0.0f;
  if (c < width) {
#pragma unroll 4
    for (int i = slice; i < rows; i += 32) v += part[(int64_t)i * width + c];
  }
  s[slice][threadIdx.x & 31] = v;
  __syncthreads();
  if (slice || c >= width) return;
  for (int i = 1; i < 32; ++i) v += s[i][threadIdx.x];
  if (c >= N) {
    if (g_pre) g_pre[c - N] = v;
  } else {
    if (g_post) g_post[c] = scale ? scale[c] * v : v;
    if (g_scale) g_scale[c] = w_post ? w_post[c] * v : v;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

// Threads of a row, eight channels each.
int row_threads(int64_t N) {
  return N <= 256 ? 32 : N <= 1024 ? 128 : N <= 2048 ? 256 : N <= 4096 ? 512 : 1024;
}

// Blocks for M rows with `threads` of them on an SM; from the shape alone, so
// that a shape always sums in the same order.
int64_t blocks_for(int64_t M, int64_t N, int threads) {
  const int tpr = row_threads(N), block = tpr == 32 ? 256 : tpr;
  const int64_t resident = (int64_t)kSms * (threads > block ? threads / block : 1);
  return least(resident, tpr == 32 ? (M + 7) / 8 : M);
}
int64_t bwd_blocks(int64_t M, int64_t N) { return blocks_for(M, N, 512); }

snn_status_t check_desc(const snn_norm_desc* d) {
  if (!d || d->reserved[0] || d->reserved[1]) return SNN_ERR_INVALID_ARG;
  if (d->M < 0 || d->N < 1 || d->group < 0) return SNN_ERR_INVALID_ARG;
  if (d->dtype < SNN_F32 || d->dtype > SNN_F16 || d->res_dtype < SNN_F32 || d->res_dtype > SNN_F16)
    return SNN_ERR_INVALID_ARG;
  if (d->gate < SNN_GATE_NONE || d->gate > SNN_GATE_SILU) return SNN_ERR_INVALID_ARG;
  if (!(d->eps > 0.0f) || !std::isfinite(d->eps)) return SNN_ERR_INVALID_ARG;
  if (d->group && d->N % d->group) return SNN_ERR_INVALID_ARG;
  if (d->N > kMaxN || d->M > (int64_t(1) << 40)) return SNN_ERR_UNSUPPORTED;
  if (d->res_dtype != SNN_F32 && d->res_dtype != d->dtype) return SNN_ERR_UNSUPPORTED;
  if (d->group && d->group != d->N &&
      (d->group < 8 || d->group > 256 || (d->group & (d->group - 1))))
    return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

const void* data_of(const snn_rows* x) { return x ? x->data : nullptr; }

// A matrix that may be absent; *vec is cleared where its rows are not whole
// 16-byte vectors.
snn_status_t take(const snn_norm_desc* d, const snn_rows* x, int dtype, Rows* out, bool* vec) {
  *out = Rows{nullptr, 0};
  if (!data_of(x)) return SNN_OK;
  if (!aligned16(x->data)) return SNN_ERR_ALIGNMENT;
  if (d->M > 1 && (x->ld < d->N || x->ld > (int64_t(1) << 40))) return SNN_ERR_INVALID_ARG;
  if (d->M > 1 && x->ld % 8) *vec = false;
  if (dtype == SNN_F32 && (reinterpret_cast<uintptr_t>(x->data) & 31u)) *vec = false;
  *out = Rows{x->data, x->ld};
  return SNN_OK;
}

struct Launch {
  const Args& g;
  bool bwd;
  int64_t blocks;
  cudaStream_t st;
};

template <typename T, typename R, bool VEC, int TPR>
cudaError_t launch_tpr(const Launch& l) {
  const dim3 grid((unsigned)l.blocks), block(kBlockThreads<TPR>);
  if (!l.bwd) return launch_pdl(norm_fwd<T, R, VEC, TPR>, grid, block, 0, l.st, l.g);
  const size_t smem = TPR == 1024 ? 4 * E * sizeof(float) * TPR : 0;
  const cudaError_t e = ensure_smem((const void*)norm_bwd<T, R, VEC, TPR>, smem);
  if (e != cudaSuccess) return e;
  return launch_pdl(norm_bwd<T, R, VEC, TPR>, grid, block, smem, l.st, l.g);
}

template <typename T, typename R, bool VEC>
cudaError_t launch_vec(const Launch& l) {
  switch (row_threads(l.g.N)) {
    case 32: return launch_tpr<T, R, VEC, 32>(l);
    case 128: return launch_tpr<T, R, VEC, 128>(l);
    case 256: return launch_tpr<T, R, VEC, 256>(l);
    case 512: return launch_tpr<T, R, VEC, 512>(l);
    default: return launch_tpr<T, R, VEC, 1024>(l);
  }
}

template <typename T, typename R>
cudaError_t launch_types(const Launch& l, bool vec) {
  return vec ? launch_vec<T, R, true>(l) : launch_vec<T, R, false>(l);
}

cudaError_t launch(const snn_norm_desc* d, const Launch& l, bool vec) {
  if (d->dtype == SNN_F32) return launch_types<float, float>(l, vec);
  if (d->dtype == SNN_BF16)
    return d->res_dtype == SNN_F32 ? launch_types<__nv_bfloat16, float>(l, vec)
                                   : launch_types<__nv_bfloat16, __nv_bfloat16>(l, vec);
  return d->res_dtype == SNN_F32 ? launch_types<__half, float>(l, vec)
                                 : launch_types<__half, __half>(l, vec);
}

Args base_args(const snn_norm_desc* d, const float* w_post, const float* scale, const float* w_pre) {
  Args g = {};
  g.M = d->M;
  g.N = (int)d->N;
  g.group = d->group ? (int)d->group : g.N;
  g.gate = d->gate;
  g.eps = d->eps;
  g.w_post = w_post;
  g.scale = scale;
  g.w_pre = w_pre;
  return g;
}

// Rows move in vectors when N and every row stride are whole ones.
snn_status_t finish(const snn_norm_desc* d, bool* vec) {
  if (d->N % 8) *vec = false;
  if (!*vec && d->group && d->group != d->N) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

}  // namespace norm
}  // namespace snn

using namespace snn::norm;

extern "C" {

size_t snn_norm_desc_size(void) { return sizeof(snn_norm_desc); }

size_t snn_block_norm_workspace_bytes(int64_t M, int64_t N) {
  if (M < 0 || N < 1 || N > kMaxN) return 0;
  const size_t b = (size_t)bwd_blocks(M, N) * 2 * (size_t)N * sizeof(float);
  return b < 256 ? 256 : b;
}

snn_status_t snn_block_norm_fwd(const snn_norm_desc* desc, const snn_rows* r, const snn_rows* a,
                                const snn_rows* z, const float* w_post, const float* res_scale,
                                const float* w_pre, const snn_rows* r_out, const snn_rows* y,
                                snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  if (desc->M == 0) return SNN_OK;
  const bool block = data_of(a) != nullptr;
  if (!data_of(r) || block != (data_of(r_out) != nullptr)) return SNN_ERR_INVALID_ARG;
  if ((w_pre != nullptr) != (data_of(y) != nullptr) || (!block && !w_pre)) return SNN_ERR_INVALID_ARG;
  if ((data_of(z) != nullptr) != (block && desc->gate != SNN_GATE_NONE)) return SNN_ERR_INVALID_ARG;
  const void* ptrs[3] = {w_post, res_scale, w_pre};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  Args g = base_args(desc, w_post, res_scale, w_pre);
  bool vec = true;
  const int io = desc->dtype, res = desc->res_dtype;
  if ((s = take(desc, r, res, &g.r, &vec)) != SNN_OK || (s = take(desc, a, io, &g.a, &vec)) != SNN_OK ||
      (s = take(desc, z, io, &g.z, &vec)) != SNN_OK || (s = take(desc, r_out, res, &g.ro, &vec)) != SNN_OK ||
      (s = take(desc, y, io, &g.y, &vec)) != SNN_OK || (s = finish(desc, &vec)) != SNN_OK)
    return s;
  const Launch l{g, false, blocks_for(desc->M, desc->N, 1024), reinterpret_cast<cudaStream_t>(stream)};
  return launch(desc, l, vec) == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

snn_status_t snn_block_norm_bwd(const snn_norm_desc* desc, const snn_rows* r_out,
                                const snn_rows* a, const snn_rows* z, const float* w_post,
                                const float* res_scale, const float* w_pre,
                                const snn_rows* grad_r_out, const snn_rows* grad_y,
                                const snn_rows* grad_r, const snn_rows* grad_a,
                                const snn_rows* grad_z, float* grad_w_post, float* grad_scale,
                                float* grad_w_pre, void* ws, size_t ws_bytes, snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  const bool block = data_of(a) != nullptr, pre = data_of(grad_y) != nullptr;
  const bool params = grad_w_post || grad_scale || grad_w_pre;
  if (desc->M > 0) {
    if (!pre && !data_of(grad_r_out)) return SNN_ERR_INVALID_ARG;
    if (pre && (!w_pre || !data_of(r_out))) return SNN_ERR_INVALID_ARG;
    if ((data_of(z) != nullptr) != (block && desc->gate != SNN_GATE_NONE)) return SNN_ERR_INVALID_ARG;
    if (!block && (data_of(grad_a) || grad_w_post || grad_scale)) return SNN_ERR_INVALID_ARG;
    if (!data_of(z) && data_of(grad_z)) return SNN_ERR_INVALID_ARG;
  }
  const void* ptrs[7] = {w_post, res_scale, w_pre, grad_w_post, grad_scale, grad_w_pre, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  if (params && (!ws || ws_bytes < snn_block_norm_workspace_bytes(desc->M, desc->N)))
    return SNN_ERR_WORKSPACE;
  Args g = base_args(desc, w_post, res_scale, w_pre);
  bool vec = true;
  const int io = desc->dtype, res = desc->res_dtype;
  if ((s = take(desc, r_out, res, &g.ro, &vec)) != SNN_OK || (s = take(desc, a, io, &g.a, &vec)) != SNN_OK ||
      (s = take(desc, z, io, &g.z, &vec)) != SNN_OK ||
      (s = take(desc, grad_r_out, res, &g.gro, &vec)) != SNN_OK ||
      (s = take(desc, grad_y, io, &g.gy, &vec)) != SNN_OK || (s = take(desc, grad_r, res, &g.gr, &vec)) != SNN_OK ||
      (s = take(desc, grad_a, io, &g.ga, &vec)) != SNN_OK || (s = take(desc, grad_z, io, &g.gz, &vec)) != SNN_OK ||
      (s = finish(desc, &vec)) != SNN_OK)
    return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const int64_t blocks = bwd_blocks(desc->M, desc->N);
  cudaError_t e = cudaSuccess;
  if (desc->M > 0) {
    g.part = params ? static_cast<float*>(ws) : nullptr;
    const Launch l{g, true, blocks, st};
    e = launch(desc, l, vec);
  }
  if (e == cudaSuccess && params)
    e = snn::launch_pdl(norm_sum, dim3((unsigned)((2 * desc->N + 31) / 32)), dim3(1024), 0, st,
                        static_cast<const float*>(ws), (int)blocks, (int)desc->N, w_post,
                        res_scale, grad_w_post, grad_scale, grad_w_pre);
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

}  // extern "C"
