// Block norms: the norm after a block, its gate and residual scale, the
// residual sum and the norm before the next block, per row of N channels:
//   n  = a rstd_a w_post            rstd_a = rsqrt(mean over the group of a^2 + eps)
//   r' = r + s n act(z)
//   y  = r' rstd w_pre              rstd   = rsqrt(mean over the row of r'^2 + eps)
// and the gradients (g = grad_y w_pre, e = r' rstd):
//   d      = grad_r' + rstd (g - e mean(g e))
//   grad_r = d;  grad_z = d s n act'(z)
//   grad_a = rstd_a (m - h mean_group(m h)),  h = a rstd_a,  m = d s act(z) w_post
//   grad_w_post = sum d s act(z) h;  grad_s = sum d n act(z);  grad_w_pre = sum grad_y e
// Every tensor is read and written once: the bound is HBM.  A row stays in
// the registers of one warp (short rows) or one block; the parameters and
// their gradients' partial sums stay in the registers of the thread that owns
// the columns, over all the rows its block takes, so the sums over rows need
// one [blocks, 3, N] array of partials and a second kernel that adds them in
// block order (no atomics: the same bits on every call).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "launch.cuh"
#include "snn.h"
#include "snn_device.cuh"

namespace snn {
namespace norm {

constexpr int64_t kMaxN = 8192;
constexpr int kMaxThreads = 512;
// Blocks whose partial sums of the parameter gradients are added: a
// constant, so that a shape always sums in the same order.
constexpr int64_t kBwdBlocks = 304;

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
  float* part;                // [blocks][3][N]
};

__device__ __forceinline__ float sigmoidf_(float z) { return 1.0f / (1.0f + __expf(-z)); }

// Element e of thread t's share of a row: eight consecutive ones per vector
// (VEC), else every TPR-th.
template <bool VEC, int TPR>
__device__ __forceinline__ int column(int t, int e) {
  return VEC ? ((e >> 3) * TPR + t) * 8 + (e & 7) : e * TPR + t;
}

template <typename T, bool VEC, int TPR, int E>
__device__ __forceinline__ void load_row(const Rows& x, int64_t row, int N, int t, float v[E]) {
  const T* p = static_cast<const T*>(x.data) + row * x.ld;
  if constexpr (VEC) {
#pragma unroll
    for (int j = 0; j < E / 8; ++j) {
      const int c = (j * TPR + t) * 8;
      if (c < N) {
        Elem<T>::load8(p + c, v + 8 * j);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[8 * j + i] = 0.0f;
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e * TPR + t < N ? Elem<T>::load1(p + e * TPR + t) : 0.0f;
  }
}

template <typename T, bool VEC, int TPR, int E>
__device__ __forceinline__ void store_row(const Rows& x, int64_t row, int N, int t, const float v[E]) {
  T* p = static_cast<T*>(x.data) + row * x.ld;
  if constexpr (VEC) {
#pragma unroll
    for (int j = 0; j < E / 8; ++j) {
      const int c = (j * TPR + t) * 8;
      if (c < N) Elem<T>::store8(p + c, v + 8 * j);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e * TPR + t < N) Elem<T>::store1(p + e * TPR + t, v[e]);
  }
}

// A parameter's share (ones where it is absent, zero past N).
template <bool VEC, int TPR, int E>
__device__ __forceinline__ void load_param(const float* p, int N, int t, float v[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int c = column<VEC, TPR>(t, e);
    v[e] = c < N ? (p ? p[c] : 1.0f) : 0.0f;
  }
}

// Sums of two values over the TPR threads of a row; every thread gets them.
template <int TPR>
__device__ __forceinline__ float2 row_sum(float2 v, float2* scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  if constexpr (TPR > 32) {
    constexpr int W = TPR / 32;
    __syncthreads();  // the last call's reads are done
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int w = 1; w < W; ++w) {
      v.x += scratch[w].x;
      v.y += scratch[w].y;
    }
  }
  return v;
}

// Sum over the group of `lanes` neighbouring threads that a vector lies in.
__device__ __forceinline__ float group_sum(float v, int lanes) {
  for (int o = 1; o < lanes; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Factor 1/rms of every element of a: over the row, or over its group (VEC;
// each of a thread's vectors lies in one group of group/8 threads).
template <int E>
struct Factors {
  float f[E / 8];
  __device__ __forceinline__ float at(int e) const { return f[e >> 3]; }
};

template <typename T, typename R, bool VEC, int TPR, int E>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_fwd(const Args g) {
  constexpr int kRowsPerBlock = TPR == 32 ? 8 : 1;
  __shared__ float2 scratch[TPR / 32];
  grid_dep_wait();
  const int t = threadIdx.x % TPR;
  const int64_t row0 = (int64_t)blockIdx.x * kRowsPerBlock + threadIdx.x / TPR;
  const bool whole = g.group == g.N;
  const float inv_n = 1.0f / (float)g.N, inv_g = 1.0f / (float)g.group;
  for (int64_t row = row0; row < g.M; row += (int64_t)gridDim.x * kRowsPerBlock) {
    float x[E], w[E];
    load_row<R, VEC, TPR, E>(g.r, row, g.N, t, x);
    if (g.a.data) {
      float a[E];
      load_row<T, VEC, TPR, E>(g.a, row, g.N, t, a);
      Factors<E> rs;
      if (whole) {
        float2 ss = make_float2(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < E; ++e) ss.x = fmaf(a[e], a[e], ss.x);
        ss = row_sum<TPR>(ss, scratch);
#pragma unroll
        for (int j = 0; j < E / 8; ++j) rs.f[j] = rsqrtf(fmaf(ss.x, inv_n, g.eps));
      } else {
#pragma unroll
        for (int j = 0; j < E / 8; ++j) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) ss = fmaf(a[8 * j + i], a[8 * j + i], ss);
          rs.f[j] = rsqrtf(fmaf(group_sum(ss, g.group >> 3), inv_g, g.eps));
        }
      }
      load_param<VEC, TPR, E>(g.w_post, g.N, t, w);
#pragma unroll
      for (int e = 0; e < E; ++e) a[e] = a[e] * rs.at(e) * w[e];
      load_param<VEC, TPR, E>(g.scale, g.N, t, w);
      if (g.z.data) {
        float z[E];
        load_row<T, VEC, TPR, E>(g.z, row, g.N, t, z);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float sg = sigmoidf_(z[e]);
          a[e] *= g.gate == SNN_GATE_SILU ? z[e] * sg : sg;
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = fmaf(w[e], a[e], x[e]);
      store_row<R, VEC, TPR, E>(g.ro, row, g.N, t, x);
    }
    if (g.y.data) {
      float2 ss = make_float2(0.f, 0.f);
#pragma unroll
      for (int e = 0; e < E; ++e) ss.x = fmaf(x[e], x[e], ss.x);
      ss = row_sum<TPR>(ss, scratch);
      const float rstd = rsqrtf(fmaf(ss.x, inv_n, g.eps));
      load_param<VEC, TPR, E>(g.w_pre, g.N, t, w);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = x[e] * rstd * w[e];
      store_row<T, VEC, TPR, E>(g.y, row, g.N, t, x);
    }
  }
}

template <typename T, typename R, bool VEC, int TPR, int E>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_bwd(const Args g) {
  constexpr int kRowsPerBlock = TPR == 32 ? 8 : 1;
  __shared__ float2 scratch[TPR / 32];
  grid_dep_wait();
  const int t = threadIdx.x % TPR;
  const int64_t row0 = (int64_t)blockIdx.x * kRowsPerBlock + threadIdx.x / TPR;
  const bool whole = g.group == g.N;
  const float inv_n = 1.0f / (float)g.N, inv_g = 1.0f / (float)g.group;
  float d_post[E], d_scale[E], d_pre[E];
#pragma unroll
  for (int e = 0; e < E; ++e) d_post[e] = d_scale[e] = d_pre[e] = 0.0f;
  for (int64_t row = row0; row < g.M; row += (int64_t)gridDim.x * kRowsPerBlock) {
    float d[E], w[E];
    if (g.gro.data) {
      load_row<R, VEC, TPR, E>(g.gro, row, g.N, t, d);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = 0.0f;
    }
    if (g.gy.data) {
      float x[E], gy[E];
      load_row<R, VEC, TPR, E>(g.ro, row, g.N, t, x);
      load_row<T, VEC, TPR, E>(g.gy, row, g.N, t, gy);
      load_param<VEC, TPR, E>(g.w_pre, g.N, t, w);
      float2 ss = make_float2(0.f, 0.f);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        ss.x = fmaf(x[e], x[e], ss.x);
        ss.y = fmaf(gy[e] * w[e], x[e], ss.y);
      }
      ss = row_sum<TPR>(ss, scratch);
      const float rstd = rsqrtf(fmaf(ss.x, inv_n, g.eps));
      const float mean = ss.y * rstd * inv_n;  // mean of (grad_y w_pre) e
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float h = x[e] * rstd;
        d[e] = fmaf(rstd, fmaf(-h, mean, gy[e] * w[e]), d[e]);
        d_pre[e] = fmaf(gy[e], h, d_pre[e]);
      }
    }
    if (g.gr.data) store_row<R, VEC, TPR, E>(g.gr, row, g.N, t, d);
    if (!g.a.data) continue;
    float a[E], sc[E];
    load_row<T, VEC, TPR, E>(g.a, row, g.N, t, a);
    load_param<VEC, TPR, E>(g.w_post, g.N, t, w);
    load_param<VEC, TPR, E>(g.scale, g.N, t, sc);
    Factors<E> rs;
    float2 ss = make_float2(0.f, 0.f);
#pragma unroll
    for (int e = 0; e < E; ++e) ss.x = fmaf(a[e], a[e], ss.x);
    if (whole) {
      ss = row_sum<TPR>(ss, scratch);
#pragma unroll
      for (int j = 0; j < E / 8; ++j) rs.f[j] = rsqrtf(fmaf(ss.x, inv_n, g.eps));
    } else {
#pragma unroll
      for (int j = 0; j < E / 8; ++j) {
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) q = fmaf(a[8 * j + i], a[8 * j + i], q);
        rs.f[j] = rsqrtf(fmaf(group_sum(q, g.group >> 3), inv_g, g.eps));
      }
    }
    // a <- h = a rstd_a;  d <- m = d s act w_post
    if (g.z.data) {
      float z[E];
      load_row<T, VEC, TPR, E>(g.z, row, g.N, t, z);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float sg = sigmoidf_(z[e]);
        const float act = g.gate == SNN_GATE_SILU ? z[e] * sg : sg;
        const float slope = g.gate == SNN_GATE_SILU ? sg * fmaf(z[e], 1.0f - sg, 1.0f) : sg * (1.0f - sg);
        a[e] *= rs.at(e);
        const float n = a[e] * w[e];
        z[e] = d[e] * sc[e] * n * slope;
        d_scale[e] = fmaf(d[e], n * act, d_scale[e]);
        const float dn = d[e] * sc[e] * act;
        d_post[e] = fmaf(dn, a[e], d_post[e]);
        d[e] = dn * w[e];
      }
      if (g.gz.data) store_row<T, VEC, TPR, E>(g.gz, row, g.N, t, z);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        a[e] *= rs.at(e);
        d_scale[e] = fmaf(d[e], a[e] * w[e], d_scale[e]);
        const float dn = d[e] * sc[e];
        d_post[e] = fmaf(dn, a[e], d_post[e]);
        d[e] = dn * w[e];
      }
    }
    if (!g.ga.data) continue;
    if (whole) {
      ss = make_float2(0.f, 0.f);
#pragma unroll
      for (int e = 0; e < E; ++e) ss.x = fmaf(d[e], a[e], ss.x);
      ss = row_sum<TPR>(ss, scratch);
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = rs.at(e) * fmaf(-a[e], ss.x * inv_n, d[e]);
    } else {
#pragma unroll
      for (int j = 0; j < E / 8; ++j) {
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) q = fmaf(d[8 * j + i], a[8 * j + i], q);
        q = group_sum(q, g.group >> 3) * inv_g;
#pragma unroll
        for (int i = 0; i < 8; ++i) d[8 * j + i] = rs.f[j] * fmaf(-a[8 * j + i], q, d[8 * j + i]);
      }
    }
    store_row<T, VEC, TPR, E>(g.ga, row, g.N, t, d);
  }
  if (!g.part) return;
  // one row of partials per row team
  float* p = g.part + ((int64_t)blockIdx.x * kRowsPerBlock + threadIdx.x / TPR) * 3 * g.N;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int c = column<VEC, TPR>(t, e);
    if (c < g.N) {
      p[c] = d_post[e];
      p[g.N + c] = d_scale[e];
      p[2 * g.N + c] = d_pre[e];
    }
  }
}

// Column sums of the partials, in row order within each of 8 slices, then
// over the slices in order.
__global__ void __launch_bounds__(256) norm_sum(const float* __restrict__ part, int rows, int N,
                                                float* o0, float* o1, float* o2) {
  __shared__ float s[8][32];
  grid_dep_wait();
  const int64_t c = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
  const int slice = threadIdx.x >> 5;
  const int64_t width = 3 * (int64_t)N;
  float v = 0.0f;
  if (c < width)
    for (int i = slice; i < rows; i += 8) v += part[i * width + c];
  s[slice][threadIdx.x & 31] = v;
  __syncthreads();
  if (slice || c >= width) return;
  for (int i = 1; i < 8; ++i) v += s[i][threadIdx.x];
  float* o = c < N ? o0 : (c < 2 * (int64_t)N ? o1 : o2);
  if (o) o[c % N] = v;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

int64_t bwd_teams(int64_t M, int64_t N) {
  // one team of 32 threads per row up to 256 channels, eight teams a block
  if (N <= 256) return least(kBwdBlocks, (M + 7) / 8) * 8;
  return least(kBwdBlocks, M);
}

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
  const int64_t per = dtype == SNN_F32 ? 4 : 8;
  if (d->M > 1 && x->ld % per) *vec = false;
  *out = Rows{x->data, x->ld};
  return SNN_OK;
}

struct Launch {
  const Args& g;
  bool bwd;
  int64_t blocks;
  cudaStream_t st;
};

template <typename T, typename R, bool VEC, int TPR, int E>
cudaError_t launch_tpr(const Launch& l) {
  const dim3 block(TPR == 32 ? 256 : TPR);
  if (l.bwd) return launch_pdl(norm_bwd<T, R, VEC, TPR, E>, dim3((unsigned)l.blocks), block, 0, l.st, l.g);
  return launch_pdl(norm_fwd<T, R, VEC, TPR, E>, dim3((unsigned)l.blocks), block, 0, l.st, l.g);
}

// Threads of a row: eight elements each, sixteen above 4096 channels.
template <typename T, typename R, bool VEC>
cudaError_t launch_vec(const Launch& l) {
  const int N = l.g.N;
  if (N <= 256) return launch_tpr<T, R, VEC, 32, 8>(l);
  if (N <= 1024) return launch_tpr<T, R, VEC, 128, 8>(l);
  if (N <= 2048) return launch_tpr<T, R, VEC, 256, 8>(l);
  if (N <= 4096) return launch_tpr<T, R, VEC, 512, 8>(l);
  return launch_tpr<T, R, VEC, 512, 16>(l);
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
  const size_t b = (size_t)bwd_teams(M, N) * 3 * (size_t)N * sizeof(float);
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
  const int64_t teams = desc->N <= 256 ? (desc->M + 7) / 8 : desc->M;
  const Launch l{g, false, least(teams, 152 * 32), reinterpret_cast<cudaStream_t>(stream)};
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
  const int64_t teams = bwd_teams(desc->M, desc->N);
  cudaError_t e = cudaSuccess;
  if (desc->M > 0) {
    g.part = params ? static_cast<float*>(ws) : nullptr;
    const Launch l{g, true, desc->N <= 256 ? teams / 8 : teams, st};
    e = launch(desc, l, vec);
  }
  if (e == cudaSuccess && params)
    e = snn::launch_pdl(norm_sum, dim3((unsigned)((3 * desc->N + 31) / 32)), dim3(256), 0, st,
                        static_cast<const float*>(ws), (int)teams, (int)desc->N, grad_w_post,
                        grad_scale, grad_w_pre);
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

}  // extern "C"
