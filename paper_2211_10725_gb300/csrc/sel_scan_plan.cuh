// How a selective scan's axis is cut, from the shape alone.
#pragma once

#include "sel_scan.cuh"

namespace snn {
namespace sscan {

constexpr int kSms = 152;

// Channel pairs of tokens that a thread of a warp loads for a tile, for PT threads of a
// pair (0: any number).
__host__ __device__ constexpr int units_of(int PT) {
  return PT == 0 ? kTile : (kTile + 32 / (32 / PT) - 1) / (32 / (32 / PT));
}

// Sum of the parts that the P threads of a pair left side by side.
template <int PT>
__device__ __forceinline__ float2 sum_parts(const float2* p, int P) {
  if constexpr (PT == 4) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    return add2(add2(make_float2(a.x, a.y), make_float2(a.z, a.w)), add2(make_float2(b.x, b.y), make_float2(b.z, b.w)));
  } else {
    float2 v = p[0];
    for (int i = 1; i < P; ++i) v = add2(v, p[i]);
    return v;
  }
}

// Cuts for `warps` warps of a whole axis: as many as make whole rounds of the
// `resident` warps that the GPU holds at once, of at least kMinSpan tokens.
constexpr int kMinSpan = 64, kMaxSpans = 64;
inline Plan cut(int64_t T, int64_t warps, int64_t resident, int rounds) {
  int64_t most = T / kMinSpan, best = 1;
  if (most > kMaxSpans) most = kMaxSpans;
  double used = 0.0;
  for (int r = 1; r <= rounds && warps > 0; ++r) {
    int64_t spans = r * resident / warps;
    if (spans < 1) continue;
    if (spans > most) spans = most;
    const double u = (double)(spans * warps) / (double)(ceil_div(spans * warps, resident) * resident);
    if (spans >= 1 && u > used + 0.03) used = u, best = spans;
  }
  Plan p;
  p.span = (int)round_up(T > 0 ? ceil_div(T, best) : 1, kTile);
  p.spans = T > 0 ? (int)ceil_div(T, p.span) : 1;
  return p;
}

inline Plan fwd_plan(const Args& g) {
  return cut(g.T, (int64_t)g.B * g.G * ceil_div(g.pairs, 32 / g.P), kSms * 16, 1);
}
inline size_t fwd_bytes(const Args& g, const Plan& p) {
  return p.spans > 1 ? ends_bytes(g, p.spans) + sums_bytes(g, p.spans) : 0;
}

cudaError_t launch_back_ends(const Args& g, int dtype, cudaStream_t st);

}  // namespace sscan
}  // namespace snn
