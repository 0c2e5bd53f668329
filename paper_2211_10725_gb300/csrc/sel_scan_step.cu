// Selective scan, one token for each sequence of a batch (decoding):
//   h <- exp(s A) h + s u B,   y = (sum_n C h + D u) silu(z)
// on fp32 states [num_slots, D, N] updated in place.  Each state is read and
// written once (8 bytes for an exponential and five operations), so the bound is
// HBM: neighbouring threads take neighbouring vectors of the states, of four
// sequences each, all on their way before the first is used.  The threads of a channel
// share out the sequences where inputs are made ready and the outputs finished.
//
// 192 sequences of 5120 channels, 16 states, from HBM: bf16 24.6 us (0.65 of the copy rate), fp32 29.0 (0.73);
// 256 of 4096 channels of 64 states 94.6 (0.86) and 112 (0.73).  Instructions bound it, 0.65 a clock: with the states
// in L2 the first still takes 19.1 us (18.5 without the decays' correction; when the kernel was first
// made one sequence a thread took 35, 64-bit products for the addresses 21, and without four blocks an SM, or three of fp32, it was
// 19.6 for 18.5 and 28.2 for 25.8).  One sequence of 1024 channels: 2.7 us.
#include "sel_scan.cuh"
#include "sel_scan_plan.cuh"

namespace snn {
namespace sscan {

constexpr int kStepThreads = 256;
constexpr int kSeqs = 4;  // of a thread

struct StepArgs {
  Args g;
  float* state;
};

// Decays of a single token, A with log2(e) (a large step with it would be past fp32): what the approximate power lacks (sel_scan.cuh) is all
// in its argument, as no settle() follows.
__device__ __forceinline__ float2 decay(float2 s, float2 A) {
  const float2 t = fma2(s, A, f2(kLift));
  const float2 part = make_float2(__saturatef(t.x * (-1.0f / kCap)), __saturatef(t.y * (-1.0f / kCap)));
  return ex2(fma2(mul2(part, part), f2(kUnits / kLn2), t));
}

// V states of a thread (V = 4: N is a multiple of four), L threads of a channel; with V = 1 and L =
// 32 a thread has two of up to 64
template <typename T, int V, int L>
__global__ void __launch_bounds__(kStepThreads, sizeof(T) == 4 ? 3 : 4) scan_step(const StepArgs a) {
  const Args& g = a.g;
  constexpr int kPass = V == 1 && L == 32 ? 2 : 1, U = L < kSeqs ? kSeqs / L : 1;
  grid_dep_wait();
  const int b0 = blockIdx.y * kSeqs, N = g.N, l = threadIdx.x & (L - 1);
  const int64_t c64 = ((int64_t)blockIdx.x * kStepThreads + threadIdx.x) / L;
  const bool live = c64 < g.D;
  const int c = live ? (int)c64 : 0, grp = c / g.Dg;
  int place[kSeqs];
#pragma unroll
  for (int j = 0; j < kSeqs; ++j) {
    place[j] = -1;
    if (b0 + j < g.B) place[j] = g.slots ? g.slots[b0 + j] : b0 + j;
    if (place[j] >= g.num_slots) place[j] = -1;
  }
  // addresses by one 32-bit product, or by steps, each (a place's D N states are below 2^28)
  const uint32_t row = (uint32_t)g.D * (uint32_t)N;
  float* const states = a.state + (int64_t)c * N + l * V;
  auto of_place = [&](int j) { return states + (uint64_t)(uint32_t)place[j] * row; };
  const T* const B0 = static_cast<const T*>(g.Bm.data) + b0 * g.Bm.sb + grp * g.Bm.sg + l * V;
  const T* const C0 = static_cast<const T*>(g.Cm.data) + b0 * g.Cm.sb + grp * g.Cm.sg + l * V;
  float h[kSeqs][kPass][V], A[kPass][V];
  Four<T> B4[kSeqs], C4[kSeqs];
  float B1[kSeqs][kPass], C1[kSeqs][kPass];
#pragma unroll
  for (int k = 0; k < kPass; ++k) {
    const int n = (k * L + l) * V;
    const bool in = live && n < N;
#pragma unroll
    for (int v = 0; v < V; ++v) A[k][v] = 0.0f;
    if (in) {
      if constexpr (V == 4) Elem<float>::load4(g.A + (int64_t)c * N + n, A[k]);
      else A[k][0] = g.A[(int64_t)c * N + n];
#pragma unroll
      for (int v = 0; v < V; ++v) A[k][v] *= kLog2E;
    }
    const T *pb = B0 + k * L * V, *pc = C0 + k * L * V;
#pragma unroll
    for (int j = 0; j < kSeqs; ++j, pb += g.Bm.sb, pc += g.Cm.sb) {
#pragma unroll
      for (int v = 0; v < V; ++v) h[j][k][v] = 0.0f;
      if constexpr (V == 4) B4[j].clear(), C4[j].clear();
      else B1[j][k] = C1[j][k] = 0.0f;
      if (in && place[j] >= 0) {
        const float* st = of_place(j) + k * L * V;
        if constexpr (V == 4) {
          Elem<float>::load4(st, h[j][k]);
          B4[j].load(pb, g.quads, 0);
          C4[j].load(pc, g.quads, 0);
        } else {
          h[j][k][0] = *st;
          B1[j][k] = Elem<T>::load1(pb);
          C1[j][k] = Elem<T>::load1(pc);
        }
      }
    }
  }
  // the thread's own sequences: l, l + L, ..
  float s[U], u[U], z[U];
  const float bias = live && g.bias ? g.bias[c] : 0.0f, skip = live && g.D_skip ? g.D_skip[c] : 0.0f;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int b = b0 + l + i * L;
    s[i] = u[i] = z[i] = 0.0f;
    if (live && l < kSeqs && b < g.B) {
      u[i] = Elem<T>::load1(static_cast<const T*>(g.u.data) + b * g.u.sb + c);
      s[i] = Elem<T>::load1(static_cast<const T*>(g.delta.data) + b * g.delta.sb + c);
      if (g.z.data) z[i] = Elem<T>::load1(static_cast<const T*>(g.z.data) + b * g.z.sb + c);
    }
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    s[i] += bias;
    if (g.softplus) s[i] = softplus<T>(f2(s[i]), nullptr).x;
  }
  float y[kSeqs];
#pragma unroll
  for (int j = 0; j < kSeqs; ++j) {
    float sj = s[j / L < U ? j / L : 0], xj = sj * u[j / L < U ? j / L : 0];
    if (L > 1) {
      const int from = (threadIdx.x & 31 & ~(L - 1)) | (j & (L - 1));
      sj = __shfl_sync(0xffffffffu, sj, from);
      xj = __shfl_sync(0xffffffffu, xj, from);
    }
    y[j] = 0.0f;
#pragma unroll
    for (int k = 0; k < kPass; ++k) {
      float B[V], C[V];
      if constexpr (V == 4) {
        B4[j].put(B);
        C4[j].put(C);
      } else {
        B[0] = B1[j][k], C[0] = C1[j][k];
      }
      if constexpr (V == 4) {
#pragma unroll
        for (int v = 0; v < V; v += 2) {
          const float2 a = decay(f2(sj), make_float2(A[k][v], A[k][v + 1]));
          const float2 now = fma2(a, make_float2(h[j][k][v], h[j][k][v + 1]), mul2(f2(xj), make_float2(B[v], B[v + 1])));
          h[j][k][v] = now.x;
          h[j][k][v + 1] = now.y;
          y[j] = fmaf(C[v], now.x, y[j]);
          y[j] = fmaf(C[v + 1], now.y, y[j]);
        }
      } else {
        h[j][k][0] = fmaf(decay(f2(sj), f2(A[k][0])).x, h[j][k][0], xj * B[0]);
        y[j] = fmaf(C[0], h[j][k][0], y[j]);
      }
      const int n = (k * L + l) * V;
      if (live && n < N && place[j] >= 0) {
        float* st = of_place(j) + k * L * V;
        if constexpr (V == 4) Elem<float>::store4(st, h[j][k]);
        else *st = h[j][k][0];
      }
    }
  }
  // the sums over a channel's threads: all four while more than four share them, then halves
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) {
    if (o >= kSeqs) {
#pragma unroll
      for (int j = 0; j < kSeqs; ++j) y[j] += __shfl_xor_sync(0xffffffffu, y[j], o);
    } else {
      const bool up = l & o;
#pragma unroll
      for (int j = 0; j < kSeqs; ++j) {
        if (j % (2 * o) < o && (L < kSeqs || j < 2 * o)) {
          const float give = up ? y[j] : y[j + o], keep = up ? y[j + o] : y[j];
          y[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int b = b0 + l + i * L;
    if (live && l < kSeqs && b < g.B) {
      float out = fmaf(skip, u[i], y[L < kSeqs ? i * L : 0]);
      if (g.z.data) out *= z[i] * sigmoid<T>(z[i]);
      bool used = false;
#pragma unroll
      for (int j = 0; j < kSeqs; ++j)
        if (j == l + i * L) used = place[j] >= 0;
      Elem<T>::store1(static_cast<T*>(g.y.data) + b * g.y.sb + c, used ? out : 0.0f);
    }
  }
}

template <typename T, int V, int L>
cudaError_t launch_lanes(const StepArgs& a, int lanes, cudaStream_t st) {
  if constexpr (V * L < (V == 4 ? 64 : 32))
    if (lanes > L) return launch_lanes<T, V, 2 * L>(a, lanes, st);
  const dim3 grid((unsigned)ceil_div((int64_t)a.g.D * L, kStepThreads), (unsigned)ceil_div(a.g.B, kSeqs));
  return launch_pdl(scan_step<T, V, L>, grid, dim3(kStepThreads), 0, st, a);
}

template <typename T>
cudaError_t launch_step(const StepArgs& a, cudaStream_t st) {
  if (a.g.N % 4 == 0) return launch_lanes<T, 4, 1>(a, a.g.N / 4, st);
  return launch_lanes<T, 1, 1>(a, a.g.N < 32 ? a.g.N : 32, st);
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
  if (desc->B > 65535) return SNN_ERR_UNSUPPORTED;  // a grid's second extent
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
  a.g.quads = quads(a.g, {&a.g.Bm, &a.g.Cm});
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = desc->dtype == SNN_F32    ? launch_step<float>(a, st)
                        : desc->dtype == SNN_BF16 ? launch_step<__nv_bfloat16>(a, st)
                                                  : launch_step<__half>(a, st);
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}
