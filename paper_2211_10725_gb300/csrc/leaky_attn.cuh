// Shared by the leaky-attention kernels and their entry points.
//
// A role is one run of the recurrence
//   E <- (state before the first token), then per token
//   R = E + b_t c_t^T;   out_t = scale * R^T a_t;   E <- beta R
// forwards or backwards in time.  The forward is the role (a, b, c) = (q, k,
// v) with E = beta S_in; the backward is three roles:
//   grad_q: (grad_o, v, k) forwards,   E = beta S_in^T
//   grad_v: (k, q, grad_o) backwards,  E = grad_S_out / scale
//   grad_k: (v, grad_o, q) backwards,  E = grad_S_out^T / scale
// The state after a forward role is the last R; after a backward one, the
// last E times scale (the gradient of S_in).
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "snn.h"

namespace snn {
namespace attn {

constexpr int kMaxD = 128;
constexpr int kMaxRoles = 3;

struct Tensor {
  void* data = nullptr;
  int64_t sb = 0, st = 0, sh = 0;
  int group = 1;  // query heads per head of this tensor
};

struct Role {
  Tensor a, b, c, out;
  int Da = 0, Dc = 0;      // widths of a/b and of c/out
  int rev = 0;             // tokens from the last to the first
  int out_f32 = 0;         // out holds fp32 (a query head's share of a shared head's gradient)
  const float* s_in = nullptr;  // [place][H][Dk][Dv]
  float* s_out = nullptr;
  int s_trans = 0;         // E is the transpose of the stored state
};

struct Args {
  Role role[kMaxRoles];
  int nroles = 0;
  int B = 0, T = 0, H = 0, Dk = 0, Dv = 0;
  float scale = 0.f;
  const float* beta = nullptr;
  const int32_t* seq_lens = nullptr;
  const int32_t* slots = nullptr;
  int64_t num_slots = 0;
  int* status = nullptr;
};

__device__ __forceinline__ int seq_len(const Args& g, int b) {
  if (!g.seq_lens) return g.T;
  const int n = g.seq_lens[b];
  return n < 0 ? 0 : (n > g.T ? g.T : n);
}

// Offset of sequence b, head h in a [place][H][Dk][Dv] state, or -1.
__device__ __forceinline__ int64_t state_offset(const Args& g, int b, int h) {
  const int64_t place = g.slots ? (int64_t)g.slots[b] : (int64_t)b;
  if (place < 0 || place >= g.num_slots) return -1;
  return (place * g.H + h) * (int64_t)g.Dk * g.Dv;
}

}  // namespace attn
}  // namespace snn
