// Argument checks shared by the leaky-attention entry points.
#pragma once

#include <cmath>
#include <cstdint>

#include "leaky_attn.cuh"

namespace snn {
namespace attn {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

inline snn_status_t check_desc(const snn_attn_desc* d) {
  if (!d || d->reserved[0] || d->reserved[1]) return SNN_ERR_INVALID_ARG;
  if (d->B < 0 || d->T < 0 || d->H < 1 || d->Hk < 1 || d->H % d->Hk) return SNN_ERR_INVALID_ARG;
  if (d->Dk < 1 || d->Dv < 1 || !std::isfinite(d->scale)) return SNN_ERR_INVALID_ARG;
  if (d->dtype != SNN_F32 && d->dtype != SNN_BF16 && d->dtype != SNN_F16) return SNN_ERR_INVALID_ARG;
  // the tensor cores take 16-bit operands in rows of whole 16-byte pieces
  if (d->dtype == SNN_F32 || d->Dk % 8 || d->Dv % 8 || d->Dk > kMaxD || d->Dv > kMaxD)
    return SNN_ERR_UNSUPPORTED;
  // block and token indexes are 32-bit
  constexpr int64_t kMost = int64_t(1) << 22;
  if (d->T > kMost || d->B > kMost || d->H > kMost || d->B * d->H > kMost) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

// A tensor of `heads` heads; T = 1 where the token stride is not looked at.
inline snn_status_t check_tensor(const snn_attn_desc* d, const snn_bthd* x, int64_t heads) {
  if (!x) return SNN_ERR_INVALID_ARG;
  if (d->B == 0 || d->T == 0) return SNN_OK;
  if (!x->data) return SNN_ERR_INVALID_ARG;
  if (!aligned16(x->data)) return SNN_ERR_ALIGNMENT;
  const int64_t ext[3] = {d->B, d->T, heads}, str[3] = {x->stride_b, x->stride_t, x->stride_h};
  for (int i = 0; i < 3; ++i) {
    if (ext[i] == 1) continue;
    if (str[i] <= 0 || str[i] >= (int64_t(1) << 38)) return SNN_ERR_INVALID_ARG;
    if (str[i] % 8) return SNN_ERR_ALIGNMENT;
  }
  return SNN_OK;
}

inline Tensor tensor(const snn_bthd* x, int group) {
  Tensor t;
  t.data = x->data;
  t.sb = x->stride_b;
  t.st = x->stride_t;
  t.sh = x->stride_h;
  t.group = group;
  return t;
}

}  // namespace attn
}  // namespace snn
