// Leaky attention over whole sequences: entry points and kernels.
//   S_t = beta S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t
// and its gradients, which are the same recurrence with the tensors' roles
// changed (see leaky_attn.cuh).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>

#include "launch.cuh"
#include "leaky_attn.cuh"
#include "leaky_attn_host.cuh"
#include "scan_host.cuh"

namespace snn {
namespace attn {

constexpr int kTokThreads = 128;
constexpr int kTokCols = 32;  // columns of the state one block keeps

// Token by token: a block keeps a [Da, 32] strip of one head's state, 32
// rows of one column in each thread's registers.
template <typename T>
__global__ void __launch_bounds__(kTokThreads) attn_tokens(const Args g) {
  grid_dep_wait();
  __shared__ float sa[kMaxD], sb[kMaxD], part[4][kTokCols];
  const Role& r = g.role[blockIdx.z];
  const int b = blockIdx.x / g.H, h = blockIdx.x % g.H;
  const int col = blockIdx.y * kTokCols + (threadIdx.x & 31), row0 = (threadIdx.x >> 5) * 32;
  const int len = seq_len(g, b);
  const bool live = col < r.Dc;
  const float beta = g.beta[h];
  const T* pa = static_cast<const T*>(r.a.data) + b * r.a.sb + (h / r.a.group) * r.a.sh;
  const T* pb = static_cast<const T*>(r.b.data) + b * r.b.sb + (h / r.b.group) * r.b.sh;
  const T* pc = static_cast<const T*>(r.c.data) + b * r.c.sb + (h / r.c.group) * r.c.sh;
  const int64_t out0 = b * r.out.sb + (h / r.out.group) * r.out.sh;
  const int64_t so = (r.s_in || r.s_out) ? state_offset(g, b, h) : -1;
  const int64_t srow = r.s_trans ? 1 : g.Dv, scol = r.s_trans ? g.Dv : 1;
  const float in_scale = r.rev ? 1.0f / g.scale : 1.0f;
  float E[32], R[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const bool in = live && row0 + i < r.Da && r.s_in && so >= 0;
    R[i] = in ? r.s_in[so + (row0 + i) * srow + col * scol] * in_scale : 0.0f;
    E[i] = r.rev ? R[i] : beta * R[i];
  }
  for (int n = 0; n < len; ++n) {
    const int64_t t = r.rev ? len - 1 - n : n;
    __syncthreads();
    if (threadIdx.x < r.Da) {
      sa[threadIdx.x] = (float)pa[t * r.a.st + threadIdx.x];
      sb[threadIdx.x] = (float)pb[t * r.b.st + threadIdx.x];
    }
    __syncthreads();
    const float c = live ? (float)pc[t * r.c.st + col] : 0.0f;
    float o = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if (row0 + i < r.Da) {
        R[i] = fmaf(sb[row0 + i], c, E[i]);
        o = fmaf(sa[row0 + i], R[i], o);
        E[i] = beta * R[i];
      }
    }
    part[threadIdx.x >> 5][threadIdx.x & 31] = o;
    __syncthreads();
    if (threadIdx.x < 32 && live) {
      const float v = g.scale * (part[0][threadIdx.x] + part[1][threadIdx.x] +
                                 part[2][threadIdx.x] + part[3][threadIdx.x]);
      const int64_t at = out0 + t * r.out.st + col;
      if (r.out_f32) static_cast<float*>(r.out.data)[at] = v;
      else static_cast<T*>(r.out.data)[at] = T(v);
    }
  }
  if (threadIdx.x < 32 && live) {
    for (int64_t t = len; t < g.T; ++t) {
      const int64_t at = out0 + t * r.out.st + col;
      if (r.out_f32) static_cast<float*>(r.out.data)[at] = 0.0f;
      else static_cast<T*>(r.out.data)[at] = T(0.0f);
    }
  }
  if (r.s_out && so >= 0 && live) {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if (row0 + i < r.Da)
        r.s_out[so + (row0 + i) * srow + col * scol] = r.rev ? E[i] * g.scale : R[i];
    }
  }
}

// out[b, t, hk, :] = sum over the group's query heads, in head order, of the
// fp32 shares part[b, t, h, :], rounded once.
template <typename T>
__global__ void __launch_bounds__(256) sum_group(const float* __restrict__ part, Tensor out, int Hk,
                                                 int G, int D, int64_t nt, int64_t n8) {
  grid_dep_wait();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n8) return;
  const int d8 = D / 8;
  const int d = (int)(i % d8) * 8;
  const int64_t row = i / d8;  // (b, t, hk)
  const int hk = (int)(row % Hk);
  const int64_t bt = row / Hk;
  const float* p = part + (bt * Hk + hk) * (int64_t)G * D + d;
  float s[8];
  Elem<float>::load8(p, s);
  for (int j = 1; j < G; ++j) {
    float v[8];
    Elem<float>::load8(p + (int64_t)j * D, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += v[e];
  }
  T* o = static_cast<T*>(out.data) + (bt / nt) * out.sb + (bt % nt) * out.st + hk * out.sh + d;
  Elem<T>::store8(o, s);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

template <typename T>
cudaError_t launch(const Args& g, cudaStream_t st) {
  int cols = 0;
  for (int i = 0; i < g.nroles; ++i) cols = g.role[i].Dc > cols ? g.role[i].Dc : cols;
  const dim3 grid((unsigned)(g.B * g.H), (unsigned)((cols + kTokCols - 1) / kTokCols), (unsigned)g.nroles);
  return launch_pdl(attn_tokens<T>, grid, dim3(kTokThreads), 0, st, g);
}

template <typename T>
cudaError_t launch_sum(const snn_attn_desc* d, const float* part, const snn_bthd* out, int D, cudaStream_t st) {
  const int64_t n8 = d->B * d->T * d->Hk * (D / 8);
  return launch_pdl(sum_group<T>, dim3((unsigned)((n8 + 255) / 256)), dim3(256), 0, st, part,
                    tensor(out, 1), (int)d->Hk, (int)(d->H / d->Hk), D, d->T, n8);
}

size_t share_bytes(const snn_attn_desc* d, int64_t D) {
  return d->H == d->Hk ? 0 : round256((size_t)(d->B * d->T * d->H * D) * sizeof(float));
}

Args base_args(const snn_attn_desc* d, const float* beta, const int32_t* seq_lens, void* ws) {
  Args g;
  g.B = (int)d->B;
  g.T = (int)d->T;
  g.H = (int)d->H;
  g.Dk = (int)d->Dk;
  g.Dv = (int)d->Dv;
  g.scale = d->scale;
  g.beta = beta;
  g.seq_lens = seq_lens;
  g.status = static_cast<int*>(ws);
  return g;
}

}  // namespace attn
}  // namespace snn

using namespace snn::attn;

extern "C" {

size_t snn_attn_desc_size(void) { return sizeof(snn_attn_desc); }

size_t snn_leaky_attn_workspace_bytes(const snn_attn_desc* desc, int backward) {
  if (check_desc(desc) != SNN_OK) return 0;
  return 256 + (backward ? share_bytes(desc, desc->Dk) + share_bytes(desc, desc->Dv) : 0);
}

snn_status_t snn_leaky_attn_fwd(const snn_attn_desc* desc, const snn_bthd* q, const snn_bthd* k,
                                const snn_bthd* v, const float* beta, const int32_t* seq_lens,
                                const float* state_in, float* state_out, const int32_t* slots,
                                int64_t num_slots, const snn_bthd* o, void* ws, size_t ws_bytes,
                                snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  const snn_bthd* x[4] = {q, k, v, o};
  const int64_t heads[4] = {desc->H, desc->Hk, desc->Hk, desc->H};
  for (int i = 0; i < 4; ++i)
    if ((s = check_tensor(desc, x[i], heads[i])) != SNN_OK) return s;
  if (!beta || (slots && num_slots < 0)) return SNN_ERR_INVALID_ARG;
  const void* ptrs[6] = {beta, seq_lens, state_in, state_out, slots, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  if (!ws || ws_bytes < snn_leaky_attn_workspace_bytes(desc, 0)) return SNN_ERR_WORKSPACE;
  if (desc->B == 0) return SNN_OK;
  const int G = (int)(desc->H / desc->Hk);
  Args g = base_args(desc, beta, seq_lens, ws);
  g.slots = slots;
  g.num_slots = slots ? num_slots : desc->B;
  g.nroles = 1;
  snn::attn::Role& r = g.role[0];
  r.a = tensor(q, 1);
  r.b = tensor(k, G);
  r.c = tensor(v, G);
  r.out = tensor(o, 1);
  r.Da = g.Dk;
  r.Dc = g.Dv;
  r.s_in = state_in;
  r.s_out = state_out;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = desc->dtype == SNN_BF16 ? launch<__nv_bfloat16>(g, st) : launch<__half>(g, st);
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

snn_status_t snn_leaky_attn_bwd(const snn_attn_desc* desc, const snn_bthd* q, const snn_bthd* k,
                                const snn_bthd* v, const float* beta, const int32_t* seq_lens,
                                const float* state_in, const snn_bthd* grad_o,
                                const float* grad_state_out, const snn_bthd* grad_q,
                                const snn_bthd* grad_k, const snn_bthd* grad_v,
                                float* grad_state_in, void* ws, size_t ws_bytes,
                                snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  if (desc->scale == 0.0f) return SNN_ERR_INVALID_ARG;
  const snn_bthd* x[7] = {q, k, v, grad_o, grad_q, grad_k, grad_v};
  const int64_t heads[7] = {desc->H, desc->Hk, desc->Hk, desc->H, desc->H, desc->Hk, desc->Hk};
  for (int i = 0; i < 7; ++i)
    if ((s = check_tensor(desc, x[i], heads[i])) != SNN_OK) return s;
  if (!beta || (grad_state_in && grad_state_in == grad_state_out)) return SNN_ERR_INVALID_ARG;
  const void* ptrs[6] = {beta, seq_lens, state_in, grad_state_out, grad_state_in, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  if (!ws || ws_bytes < snn_leaky_attn_workspace_bytes(desc, 1)) return SNN_ERR_WORKSPACE;
  if (desc->B == 0) return SNN_OK;
  const int G = (int)(desc->H / desc->Hk);
  Args g = base_args(desc, beta, seq_lens, ws);
  g.num_slots = desc->B;
  g.nroles = 3;
  unsigned char* at = static_cast<unsigned char*>(ws) + 256;
  float* share_k = reinterpret_cast<float*>(at);
  float* share_v = reinterpret_cast<float*>(at + share_bytes(desc, desc->Dk));
  auto share = [&](float* p, int64_t D) {
    Tensor t;
    t.data = p;
    t.sh = D;
    t.st = desc->H * D;
    t.sb = desc->T * t.st;
    return t;
  };
  snn::attn::Role& rq = g.role[0];
  rq.a = tensor(grad_o, 1);
  rq.b = tensor(v, G);
  rq.c = tensor(k, G);
  rq.out = tensor(grad_q, 1);
  rq.Da = g.Dv;
  rq.Dc = g.Dk;
  rq.s_in = state_in;
  rq.s_trans = 1;
  snn::attn::Role& rv = g.role[1];
  rv.a = tensor(k, G);
  rv.b = tensor(q, 1);
  rv.c = tensor(grad_o, 1);
  rv.out = G == 1 ? tensor(grad_v, 1) : share(share_v, desc->Dv);
  rv.Da = g.Dk;
  rv.Dc = g.Dv;
  rv.rev = 1;
  rv.s_in = grad_state_out;
  rv.s_out = grad_state_in;
  snn::attn::Role& rk = g.role[2];
  rk.a = tensor(v, G);
  rk.b = tensor(grad_o, 1);
  rk.c = tensor(q, 1);
  rk.out = G == 1 ? tensor(grad_k, 1) : share(share_k, desc->Dk);
  rk.Da = g.Dv;
  rk.Dc = g.Dk;
  rk.rev = 1;
  rk.s_in = grad_state_out;
  rk.s_trans = 1;
  rv.out_f32 = rk.out_f32 = G > 1;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const bool bf = desc->dtype == SNN_BF16;
  cudaError_t e = bf ? launch<__nv_bfloat16>(g, st) : launch<__half>(g, st);
  if (e == cudaSuccess && G > 1 && desc->T > 0) {
    e = bf ? launch_sum<__nv_bfloat16>(desc, share_k, grad_k, g.Dk, st)
           : launch_sum<__half>(desc, share_k, grad_k, g.Dk, st);
    if (e == cudaSuccess)
      e = bf ? launch_sum<__nv_bfloat16>(desc, share_v, grad_v, g.Dv, st)
             : launch_sum<__half>(desc, share_v, grad_v, g.Dv, st);
  }
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

}  // extern "C"
