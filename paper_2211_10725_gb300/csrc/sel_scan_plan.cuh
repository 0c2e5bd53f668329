// How a selective scan's axis is cut, from the shape alone.
#pragma once

#include "sel_scan.cuh"

namespace snn {
namespace sscan {

constexpr int kThreads = 128;
constexpr int kSms = 152;

// Tokens of a forward tile: at most four channel pairs of tokens to a thread.
__host__ __device__ constexpr int tile_tokens(int P) { return P >= 4 ? 16 : P >= 2 ? 8 : 4; }

// Cuts so that `blocks` blocks become about `target`, each of at least kMinSpan tokens.
constexpr int kMinSpan = 64, kMaxSpans = 64;
inline Plan cut(int64_t T, int64_t blocks, int64_t target) {
  int64_t spans = blocks > 0 ? target / blocks : 1;
  if (spans > T / kMinSpan) spans = T / kMinSpan;
  if (spans > kMaxSpans) spans = kMaxSpans;
  if (spans < 1) spans = 1;
  Plan p;
  p.span = (int)round_up(T > 0 ? ceil_div(T, spans) : 1, 16);
  p.spans = T > 0 ? (int)ceil_div(T, p.span) : 1;
  return p;
}

inline Plan fwd_plan(const Args& g) {
  const int64_t blocks = (int64_t)g.B * g.G * ceil_div(g.pairs, kThreads / g.P);
  return cut(g.T, blocks, kSms * 6);
}
inline size_t fwd_bytes(const Args& g, const Plan& p) {
  return p.spans > 1 ? ends_bytes(g, p.spans) + sums_bytes(g, p.spans) : 0;
}

cudaError_t launch_back_ends(const Args& g, int dtype, cudaStream_t st);

}  // namespace sscan
}  // namespace snn
