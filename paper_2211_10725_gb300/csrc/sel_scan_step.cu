// Selective scan, one token for each sequence of a batch (decoding):
//   h <- exp(s A) h + s u B,   y = (sum_n C h + D u) silu(z)
// on fp32 states [num_slots, D, N] updated in place.  Each state is read and
// written once (8 bytes for an exponential and five operations), so the bound is
// HBM: neighbouring threads take neighbouring vectors of the states, one access
// each, and a channel's sum goes through shuffles.
#include "sel_scan.cuh"

namespace snn {
namespace sscan {

constexpr int kStepThreads = 256;

struct StepArgs {
  Args g;
  int lanes;     // threads of a channel, a power of two up to 32
  int bc_vec;    // B and C can be read in vectors of four
  float* state;
};

// V states of a thread; V = 4: N is a multiple of four
template <typename T, int V>
__global__ void __launch_bounds__(kStepThreads) scan_step(const StepArgs a) {
  const Args& g = a.g;
  constexpr int kPass = V == 4 ? 1 : 2;  // of V lanes states each; up to 64 states
  grid_dep_wait();
  const int b = blockIdx.y, N = g.N;
  const int lane = threadIdx.x & (a.lanes - 1);
  const int64_t c64 = ((int64_t)blockIdx.x * kStepThreads + threadIdx.x) / a.lanes;
  const int64_t place = g.slots ? (int64_t)g.slots[b] : (int64_t)b;
  const bool live = c64 < g.D, used = place >= 0 && place < g.num_slots;
  const int c = live ? (int)c64 : 0;
  T* py = static_cast<T*>(g.y.data) + b * g.y.sb + c;
  if (!used) {  // an empty place of the batch
    if (live && lane == 0) Elem<T>::store1(py, 0.0f);
    return;
  }
  float* st = a.state + (place * g.D + c) * (int64_t)N;
  const float* pa = g.A + (int64_t)c * N;
  const int grp = c / g.Dg;
  const T* pb = static_cast<const T*>(g.Bm.data) + b * g.Bm.sb + grp * g.Bm.sg;
  const T* pc = static_cast<const T*>(g.Cm.data) + b * g.Cm.sb + grp * g.Cm.sg;
  float h[kPass][V], A[kPass][V], B[kPass][V], C[kPass][V];
#pragma unroll
  for (int k = 0; k < kPass; ++k) {
    const int n = (k * a.lanes + lane) * V;
    if (live && n < N) {
      if constexpr (V == 4) {
        Elem<float>::load4(st + n, h[k]);
        Elem<float>::load4(pa + n, A[k]);
        if (a.bc_vec) {
          Elem<T>::load4(pb + n, B[k]);
          Elem<T>::load4(pc + n, C[k]);
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v) B[k][v] = Elem<T>::load1(pb + n + v), C[k][v] = Elem<T>::load1(pc + n + v);
        }
      } else {
        h[k][0] = st[n], A[k][0] = pa[n], B[k][0] = Elem<T>::load1(pb + n), C[k][0] = Elem<T>::load1(pc + n);
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) h[k][v] = A[k][v] = B[k][v] = C[k][v] = 0.0f;
    }
  }
  const float u = Elem<T>::load1(static_cast<const T*>(g.u.data) + b * g.u.sb + c);
  float s = Elem<T>::load1(static_cast<const T*>(g.delta.data) + b * g.delta.sb + c);
  float z = 0.0f;
  if (g.z.data) z = Elem<T>::load1(static_cast<const T*>(g.z.data) + b * g.z.sb + c);
  if (g.bias) s += g.bias[c];
  const float skip = g.D_skip ? g.D_skip[c] : 0.0f;
  if (g.softplus) s = softplus<T>(f2(s), nullptr).x;
  const float x = s * u, s2 = s * kLog2E;
  float y = 0.0f;
#pragma unroll
  for (int k = 0; k < kPass; ++k) {
    const int n = (k * a.lanes + lane) * V;
    if (live && n < N) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        h[k][v] = fmaf(ex2(s2 * A[k][v]), h[k][v], x * B[k][v]);
        y = fmaf(C[k][v], h[k][v], y);
      }
      if constexpr (V == 4) Elem<float>::store4(st + n, h[k]);
      else st[n] = h[k][0];
    }
  }
  for (int o = 1; o < a.lanes; o <<= 1) y += __shfl_xor_sync(0xffffffffu, y, o);
  if (live && lane == 0) {
    y = fmaf(skip, u, y);
    if (g.z.data) y *= z * sigmoid<T>(z);
    Elem<T>::store1(py, y);
  }
}

template <typename T>
cudaError_t launch_step(StepArgs a, cudaStream_t st) {
  const int vecs = a.g.N % 4 == 0 ? a.g.N / 4 : a.g.N;
  a.lanes = 1;
  while (a.lanes < vecs && a.lanes < 32) a.lanes *= 2;
  const dim3 grid((unsigned)ceil_div((int64_t)a.g.D * a.lanes, kStepThreads), (unsigned)a.g.B);
  if (a.g.N % 4 == 0) return launch_pdl(scan_step<T, 4>, grid, dim3(kStepThreads), 0, st, a);
  return launch_pdl(scan_step<T, 1>, grid, dim3(kStepThreads), 0, st, a);
}

}  // namespace sscan
}  // namespace snn

using namespace snn::sscan;

extern "C" snn_status_t snn_selective_scan_step(const snn_sscan_desc* desc, const snn_btc* u,
                                                const snn_btc* delta, const float* A,
                                                const snn_bthd* Bm, const snn_bthd* Cm,
                                                const float* D, const snn_btc* z,
                                                const float* delta_bias, float* state,
                                                const int32_t* slots, int64_t num_slots,
                                                const snn_btc* y, snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  if (desc->T != 1 || !A || !state || num_slots < 0 || num_slots > kMost) return SNN_ERR_INVALID_ARG;
  if (!slots && num_slots < desc->B) return SNN_ERR_INVALID_ARG;
  if (desc->B > 65535) return SNN_ERR_UNSUPPORTED;
  const void* ptrs[5] = {A, D, delta_bias, state, slots};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  if (desc->B == 0) return SNN_OK;
  StepArgs a = {};
  a.g = base_args(desc);
  bool pair = true;
  if ((s = take(desc, u, &a.g.u, &pair)) != SNN_OK || (s = take(desc, delta, &a.g.delta, &pair)) != SNN_OK ||
      (z && z->data && (s = take(desc, z, &a.g.z, &pair)) != SNN_OK) ||
      (s = take(desc, y, &a.g.y, &pair)) != SNN_OK || (s = take(desc, Bm, &a.g.Bm)) != SNN_OK ||
      (s = take(desc, Cm, &a.g.Cm)) != SNN_OK)
    return s;
  a.g.A = A;
  a.g.D_skip = D;
  a.g.bias = delta_bias;
  a.g.slots = slots;
  a.g.num_slots = num_slots;
  a.state = state;
  a.bc_vec = quads(a.g, {&a.g.Bm, &a.g.Cm});
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = desc->dtype == SNN_F32    ? launch_step<float>(a, st)
                        : desc->dtype == SNN_BF16 ? launch_step<__nv_bfloat16>(a, st)
                                                  : launch_step<__half>(a, st);
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}
