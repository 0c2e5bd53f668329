// Layer norm of rows of N channels:
//   e = (x - mean) rstd,   rstd = rsqrt(mean of (x - mean)^2 + eps),   y = e w + b
// and its gradients (g = grad_y w):
//   grad_x = rstd (g - mean(g) - e mean(g e));   grad_w = sum grad_y e;   grad_b = sum grad_y
// Every tensor is read and written once, so the bound is HBM.  The plan is that
// of the block norms (norm_rows.cuh): a warp or a block to a row, eight channels
// to a thread, the next two rows on their way to its registers while the present
// ones are worked on (through shared memory, 16384x4096 bf16 on an fp32 stream took 77 us
// for 70: its copies of 16 bytes each touch half a sector of a 32-bit row; three rows on
// their way 69 for 68).  Rows that are not whole 16-byte vectors, and
// the longest rows' backward, pass through shared memory.  The variance is the sum of
// squares about the mean, from the registers: a row far from zero loses no
// bits.  The backward takes mean and rstd as the forward stored them (8 bytes a
// row), so that its two sums over a row meet in one exchange; grad_w and grad_b gather
// in the registers of the channels' owners over all the rows of a block, and a second
// kernel adds the blocks in their order (no atomics: the same bits on every call).
// Now 16384x4096 bf16 on an fp32 stream takes 61 us (0.97 of the copy rate), 16384x2048 bf16
// 25 (0.8) and its backward 39 (0.77) and 5 for the sums.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "launch.cuh"
#include "norm_rows.cuh"
#include "scan_host.cuh"
#include "snn.h"
#include "snn_device.cuh"

namespace snn {
namespace lnorm {

using namespace snn::norm;
using snn::norm::add2;
using snn::norm::fma2;
using snn::norm::mul2;

struct Args {
  int64_t M;
  int N;
  float eps;
  Rows x, y;       // forward
  Rows gy, gx;     // backward (reads x)
  const float *w, *b;
  float* stats;    // [2][M]: means, reciprocal deviations
  int stages;      // rows a team has in shared memory at once, 1 to 3
  float* part;     // [blocks][2][N]: of grad_y e, of grad_y
};

__device__ __forceinline__ float sum(const float v[E]) {
  float2 s = two(v, 0);
#pragma unroll
  for (int e = 2; e < E; e += 2) s = add2(s, two(v, e));
  return s.x + s.y;
}

__host__ __device__ constexpr int bwd_stage(int N, int t_size, int r_size) {
  return slot_bytes(N, r_size) + slot_bytes(N, t_size);
}

// Rows that a team works on at once, their sums in one exchange.  Forward where
// a row is several warps' (16384x4096 bf16 on an fp32 stream: 63 us, 68 with one
// row at a time; 16384x2048 bf16: 24.8 and 27.9), but one by one where it is one
// warp's (no barrier to share: 40000x200 23.7 against 21.6, with its gradients)
// or a whole block's (8192x8192: 82.6 against 77.8).  Backward for all but the longest rows,
// whose threads have 64 registers (16384x2048 bf16: 38 us, 47).
template <int TPR>
constexpr bool kPaired = TPR > 32 && TPR < 1024;
template <int TPR>
constexpr int kBwdRows = TPR == 1024 ? 1 : 2;

extern __shared__ __align__(16) unsigned char ln_smem[];

template <typename T, typename R, bool VEC, int TPR>
__global__ void __launch_bounds__(kBlockThreads<TPR>, 1024 / kBlockThreads<TPR>) ln_fwd(const Args g) {
  __shared__ __align__(16) float scratch[2][3][32];
  grid_dep_wait();
  const int t = threadIdx.x % TPR, team = threadIdx.x / TPR, N = g.N;
  const int64_t step = (int64_t)gridDim.x * kTeams<TPR>;
  int64_t row = (int64_t)blockIdx.x * kTeams<TPR> + team;
  const float inv_n = 1.0f / (float)N;
  RowSum<TPR> row_sum{scratch};
  float w[E], b[E];
  load_param<VEC, TPR>(g.w, N, t, w);
  if (g.b) {
    load_param<VEC, TPR>(g.b, N, t, b);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) b[e] = 0.0f;
  }
  const int stage = slot_bytes(N, sizeof(R));
  unsigned char* const base = ln_smem + team * g.stages * stage;
  auto slot = [&](int k) { return Slot<R, VEC, TPR>{base + k * stage}; };
  auto fetch = [&](int64_t i, int k) {
    if (i < g.M) slot(k).fetch(g.x, i, g.M, N, t);
    copies_commit();
  };
  auto work = [&](int64_t first, auto& x) {  // x: [rows][E]
    constexpr int kRows = sizeof(x) / sizeof(x[0]);
    float s[kRows], mean[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) s[j] = sum(x[j]);
    row_sum(s);
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      mean[j] = s[j] * inv_n;
      if constexpr (VEC) {  // past N: zero less zero
        const float off = t * E < N ? -mean[j] : 0.0f;
#pragma unroll
        for (int e = 0; e < E; e += 2) put2(x[j], e, add2(two(x[j], e), both(off)));
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[j][e] = e * TPR + t < N ? x[j][e] - mean[j] : 0.0f;
      }
      s[j] = square_sum(x[j]);
    }
    row_sum(s);
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      const int64_t row = first + j * step;
      if (j && row >= g.M) break;
      const float rstd = rsqrtf(fmaf(s[j], inv_n, g.eps));
      if (g.stats && t == 0) {
        g.stats[row] = mean[j];
        g.stats[g.M + row] = rstd;
      }
#pragma unroll
      for (int e = 0; e < E; e += 2)
        put2(x[j], e, fma2(mul2(two(x[j], e), both(rstd)), two(w, e), two(b, e)));
      store_row<T, VEC, TPR>(g.y, row, N, t, x[j]);
    }
  };
  if constexpr (VEC) {
    Held<R> held[2];
    auto take = [&](int64_t i, Held<R>& h, float (&x)[E]) {  // row i, and two rows on on its way
      h.get(N, t, x);
      if (i + 2 * step < g.M) h.fetch(g.x, i + 2 * step, N, t);
    };
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (row + j * step < g.M) held[j].fetch(g.x, row + j * step, N, t);
    while (row < g.M) {
      if constexpr (kPaired<TPR>) {
        float x[2][E];  // (the second row past M: whatever its registers hold, never stored)
#pragma unroll
        for (int j = 0; j < 2; ++j) take(row + j * step, held[j], x[j]);
        work(row, x);
        row += 2 * step;
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (row < g.M) {
            float x[1][E];
            take(row, held[j], x[0]);
            work(row, x);
          }
          row += step;
        }
      }
    }
  } else {
    const int ahead = g.stages - 1;  // at least one
    for (int i = 0; i < ahead; ++i) fetch(row + i * step, i);
    for (int k = 0, next = ahead; row < g.M; row += step) {
      fetch(row + ahead * step, next);  // that stage was read before the last row's sums
      copies_wait(ahead);
      team_sync<TPR>();
      float x[1][E];
      slot(k).get(g.x, row, N, t, x[0]);
      if (TPR == 32) team_sync<TPR>();
      work(row, x);
      k = k + 1 == g.stages ? 0 : k + 1;
      next = next + 1 == g.stages ? 0 : next + 1;
    }
    copies_wait(0);
  }
}

template <typename T, typename R, bool VEC, int TPR>
__global__ void __launch_bounds__(kBlockThreads<TPR>, TPR == 1024 ? 1 : kBwdThreads / kBlockThreads<TPR>)
    ln_bwd(const Args g) {
  constexpr int kRows = kBwdRows<TPR>;
  __shared__ __align__(16) float scratch[2][2 * kRows][32];
  grid_dep_wait();
  constexpr bool kLong = TPR == 1024, kHeld = VEC && !kLong;
  const int t = threadIdx.x % TPR, team = threadIdx.x / TPR, N = g.N;
  const int64_t step = (int64_t)gridDim.x * kTeams<TPR>;
  int64_t row = (int64_t)blockIdx.x * kTeams<TPR> + team;
  const float inv_n = 1.0f / (float)N;
  RowSum<TPR, 2 * kRows> row_sum{scratch};
  const int slot_size = bwd_stage(N, sizeof(T), sizeof(R)), stage = kRows * slot_size;
  unsigned char* const base = ln_smem + team * g.stages * stage;
  const int r_bytes = slot_bytes(N, sizeof(R));
  auto x_slot = [&](int k, int j) { return Slot<R, VEC, TPR>{base + k * stage + j * slot_size}; };
  auto gy_slot = [&](int k, int j) { return Slot<T, VEC, TPR>{base + k * stage + j * slot_size + r_bytes}; };
  auto fetch = [&](int64_t i, int k) {
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      if (i + j * step < g.M) {
        x_slot(k, j).fetch(g.x, i + j * step, g.M, N, t);
        gy_slot(k, j).fetch(g.gy, i + j * step, g.M, N, t);
      }
    }
    copies_commit();
  };
  const int ahead = g.stages - 1;
  Held<R> held_x[kRows];
  Held<T> held_gy[kRows];
  float next_mean[kRows], next_rstd[kRows];
  auto hold = [&](int64_t i) {
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      if (i + j * step >= g.M) return;
      held_x[j].fetch(g.x, i + j * step, N, t);
      held_gy[j].fetch(g.gy, i + j * step, N, t);
    }
  };
  auto take_stats = [&](int64_t i) {
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      if (i + j * step >= g.M) return;
      next_mean[j] = g.stats[i + j * step];
      next_rstd[j] = g.stats[g.M + i + j * step];
    }
  };
#pragma unroll
  for (int j = 0; j < kRows; ++j) next_mean[j] = next_rstd[j] = 0.0f;
  if constexpr (kHeld) {
    hold(row);
  } else {
    for (int i = 0; i < (ahead ? ahead : 1); ++i) fetch(row + i * kRows * step, i);
  }
  take_stats(row);
  Sums<kLong> sums;  // 0: of grad_y e, 1: of grad_y
  sums.at = reinterpret_cast<float4*>(ln_smem + g.stages * stage);
  sums.threads = TPR;
  sums.clear();
  float w[E], one[E];
#pragma unroll
  for (int e = 0; e < E; ++e) one[e] = 1.0f;
  load_param<VEC, TPR>(g.w, N, t, w);
  for (int k = 0, next = ahead; row < g.M; row += kRows * step) {
    float x[kRows][E], gy[kRows][E];
    if constexpr (kHeld) {
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        held_x[j].get(N, t, x[j]);
        held_gy[j].get(N, t, gy[j]);
      }
      hold(row + kRows * step);
    } else {
      if (ahead) fetch(row + ahead * kRows * step, next);  // that stage was read before the last rows' sums
      copies_wait(ahead);
      if (!VEC) team_sync<TPR>();
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        x_slot(k, j).get(g.x, row + j * step, N, t, x[j]);
        gy_slot(k, j).get(g.gy, row + j * step, N, t, gy[j]);
      }
    }
    float mean[kRows], rstd[kRows], ss[2 * kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      mean[j] = next_mean[j];
      rstd[j] = next_rstd[j];
    }
    take_stats(row + kRows * step);
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      float v[E];
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        put2(x[j], e, mul2(add2(two(x[j], e), both(-mean[j])), both(rstd[j])));
        put2(v, e, mul2(two(gy[j], e), two(w, e)));
      }
      // past N: v is zero, so the x there enters nothing; a row past M enters no sum
      if (row + j * step < g.M) {
        sums.add(0, gy[j], x[j]);
        sums.add(1, gy[j], one);
      }
      ss[2 * j] = sum(v);
      ss[2 * j + 1] = dot(v, x[j]);
#pragma unroll
      for (int e = 0; e < E; ++e) gy[j][e] = v[e];
    }
    row_sum(ss);
    if (!VEC && TPR == 32) team_sync<TPR>();
    if (!kHeld && !ahead) fetch(row + kRows * step, 0);  // the rows are read: their stage is free
    if (g.gx.data) {
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        if (row + j * step >= g.M) break;
        const float m0 = ss[2 * j] * inv_n, m1 = ss[2 * j + 1] * inv_n;
#pragma unroll
        for (int e = 0; e < E; e += 2)
          put2(gy[j], e, mul2(both(rstd[j]), fma2(two(x[j], e), both(-m1), add2(two(gy[j], e), both(-m0)))));
        store_row<R, VEC, TPR>(g.gx, row + j * step, N, t, gy[j]);
      }
    }
    k = k + 1 == g.stages ? 0 : k + 1;
    next = next + 1 == g.stages ? 0 : next + 1;
  }
  copies_wait(0);
  if (!g.part) return;
  float* p = g.part + (int64_t)blockIdx.x * 2 * N;
  if constexpr (kTeams<TPR> > 1) {  // the block's teams, in order
    constexpr int kWidth = TPR * E;
    float* all = reinterpret_cast<float*>(ln_smem);  // [teams][2][kWidth], over the rows
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float v[E];
      sums.get(k, v);
#pragma unroll
      for (int e = 0; e < E; ++e) all[(team * 2 + k) * kWidth + (VEC ? t * E + e : e * TPR + t)] = v[e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * N; i += kBlockThreads<TPR>) {
      const int k = i / N, at = k * kWidth + i - k * N;
      float v = all[at];
#pragma unroll
      for (int j = 1; j < kTeams<TPR>; ++j) v += all[j * 2 * kWidth + at];
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
__global__ void __launch_bounds__(1024) ln_sum(const float* __restrict__ part, int rows, int N,
                                               float* grad_w, float* grad_b) {
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
    if (grad_b) grad_b[c - N] = v;
  } else if (grad_w) {
    grad_w[c] = v;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

snn_status_t check_desc(const snn_layer_norm_desc* d, bool eps) {
  if (!d || d->reserved) return SNN_ERR_INVALID_ARG;
  if (d->M < 0 || d->N < 1) return SNN_ERR_INVALID_ARG;
  if (d->dtype < SNN_F32 || d->dtype > SNN_F16 || d->res_dtype < SNN_F32 || d->res_dtype > SNN_F16)
    return SNN_ERR_INVALID_ARG;
  if (eps && (!(d->eps > 0.0f) || !std::isfinite(d->eps))) return SNN_ERR_INVALID_ARG;
  if (d->N > kMaxN || d->M > (int64_t(1) << 40)) return SNN_ERR_UNSUPPORTED;
  if (d->res_dtype != SNN_F32 && d->res_dtype != d->dtype) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

// A matrix; *vec is cleared where its rows are not whole 16-byte vectors.
snn_status_t take(const snn_layer_norm_desc* d, const snn_rows* x, Rows* out, bool* vec) {
  if (!aligned16(x->data)) return SNN_ERR_ALIGNMENT;
  if (d->M > 1 && (x->ld < d->N || x->ld > (int64_t(1) << 40))) return SNN_ERR_INVALID_ARG;
  if (d->M > 1 && x->ld % 8) *vec = false;
  *out = Rows{x->data, x->ld};
  return SNN_OK;
}

struct Launch {
  const Args& g;
  bool bwd;
  int64_t blocks;
  cudaStream_t st;
};

// Rows in shared memory: up to three, as many as fit beside the other blocks
// of an SM (and the sums of long rows).
template <typename K>
cudaError_t launch_staged(K* kernel, const Launch& l, int threads, int teams, int stage, size_t fixed,
                          int resident, int least_stages) {
  constexpr size_t kPerSm = 224 * 1024;
  Args g = l.g;
  g.stages = 3;
  while (g.stages > least_stages && g.stages * (size_t)teams * stage + fixed + 1024 > kPerSm / resident) --g.stages;
  size_t smem = g.stages * (size_t)teams * stage + fixed;
  const size_t all = teams > 1 ? (size_t)teams * 2 * 32 * E * sizeof(float) : 0;  // short rows' sums
  if (smem < all) smem = all;
  // with the kernel's static shared memory, past the limit that needs no asking
  const size_t ask = smem + 1024 > 48 * 1024 && smem <= 48 * 1024 ? 48 * 1024 + 16 : smem;
  const cudaError_t e = ensure_smem((const void*)kernel, ask);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3((unsigned)l.blocks), dim3(threads), smem, l.st, g);
}

template <typename T, typename R, bool VEC, int TPR>
cudaError_t launch_tpr(const Launch& l) {
  constexpr int kThreads = kBlockThreads<TPR>;
  if (!l.bwd)
    return launch_staged(ln_fwd<T, R, VEC, TPR>, l, kThreads, kTeams<TPR>,
                         VEC ? 0 : slot_bytes(l.g.N, sizeof(R)), 0, 1024 / kThreads, 2);
  return launch_staged(ln_bwd<T, R, VEC, TPR>, l, kThreads, kTeams<TPR>,
                       VEC && TPR < 1024 ? 0 : kBwdRows<TPR> * bwd_stage(l.g.N, sizeof(T), sizeof(R)),
                       TPR == 1024 ? 2 * E * sizeof(float) * TPR : 0,
                       TPR == 1024 ? 1 : kBwdThreads / kThreads, 1);
}

template <typename T, typename R, bool VEC>
cudaError_t launch_vec(const Launch& l) {
  switch (row_threads(l.g.N)) {
    case 32: return launch_tpr<T, R, VEC, 32>(l);
    case 64: return launch_tpr<T, R, VEC, 64>(l);
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

cudaError_t launch(const snn_layer_norm_desc* d, const Launch& l, bool vec) {
  if (d->dtype == SNN_F32) return launch_types<float, float>(l, vec);
  if (d->dtype == SNN_BF16)
    return d->res_dtype == SNN_F32 ? launch_types<__nv_bfloat16, float>(l, vec)
                                   : launch_types<__nv_bfloat16, __nv_bfloat16>(l, vec);
  return d->res_dtype == SNN_F32 ? launch_types<__half, float>(l, vec)
                                 : launch_types<__half, __half>(l, vec);
}

Args base_args(const snn_layer_norm_desc* d, const float* w, const float* b, const float* stats) {
  Args g = {};
  g.M = d->M;
  g.N = (int)d->N;
  g.eps = d->eps;
  g.w = w;
  g.b = b;
  g.stats = const_cast<float*>(stats);
  return g;
}

}  // namespace lnorm
}  // namespace snn

using namespace snn::lnorm;

extern "C" {

size_t snn_layer_norm_desc_size(void) { return sizeof(snn_layer_norm_desc); }

size_t snn_layer_norm_workspace_bytes(int64_t M, int64_t N) {
  if (M < 0 || N < 1 || N > snn::norm::kMaxN) return 0;
  const size_t b = (size_t)bwd_blocks(M, N) * 2 * (size_t)N * sizeof(float);
  return b < 256 ? 256 : b;
}

snn_status_t snn_layer_norm_fwd(const snn_layer_norm_desc* desc, const snn_rows* x, const float* w,
                                const float* b, const snn_rows* y, float* stats, snn_stream_t stream) {
  snn_status_t s = check_desc(desc, true);
  if (s != SNN_OK) return s;
  if (desc->M == 0) return SNN_OK;
  if (!data_of(x) || !data_of(y)) return SNN_ERR_INVALID_ARG;
  const void* ptrs[3] = {w, b, stats};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  Args g = base_args(desc, w, b, stats);
  bool vec = desc->N % 8 == 0;
  if ((s = take(desc, x, &g.x, &vec)) != SNN_OK || (s = take(desc, y, &g.y, &vec)) != SNN_OK) return s;
  const Launch l{g, false, blocks_for(desc->M, desc->N, 1024), reinterpret_cast<cudaStream_t>(stream)};
  return launch(desc, l, vec) == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

snn_status_t snn_layer_norm_bwd(const snn_layer_norm_desc* desc, const snn_rows* x, const float* w,
                                const float* stats, const snn_rows* grad_y, const snn_rows* grad_x,
                                float* grad_w, float* grad_b, void* ws, size_t ws_bytes,
                                snn_stream_t stream) {
  snn_status_t s = check_desc(desc, false);
  if (s != SNN_OK) return s;
  const bool params = grad_w || grad_b;
  if (desc->M > 0 && (!data_of(x) || !stats || !data_of(grad_y))) return SNN_ERR_INVALID_ARG;
  const void* ptrs[5] = {w, stats, grad_w, grad_b, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  if (params && (!ws || ws_bytes < snn_layer_norm_workspace_bytes(desc->M, desc->N))) return SNN_ERR_WORKSPACE;
  Args g = base_args(desc, w, nullptr, stats);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const int64_t blocks = bwd_blocks(desc->M, desc->N);
  cudaError_t e = cudaSuccess;
  if (desc->M > 0) {
    bool vec = desc->N % 8 == 0;
    if ((s = take(desc, x, &g.x, &vec)) != SNN_OK || (s = take(desc, grad_y, &g.gy, &vec)) != SNN_OK ||
        (data_of(grad_x) && (s = take(desc, grad_x, &g.gx, &vec)) != SNN_OK))
      return s;
    g.part = params ? static_cast<float*>(ws) : nullptr;
    const Launch l{g, true, blocks, st};
    if (params || data_of(grad_x)) e = launch(desc, l, vec);
  }
  if (e == cudaSuccess && params)
    e = snn::launch_pdl(ln_sum, dim3((unsigned)((2 * desc->N + 31) / 32)), dim3(1024), 0, st,
                        static_cast<const float*>(ws), (int)blocks, (int)desc->N, grad_w, grad_b);
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

}  // extern "C"
