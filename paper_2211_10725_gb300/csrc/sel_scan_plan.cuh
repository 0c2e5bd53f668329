// How a selective scan is laid on threads and its axis cut, from the shape alone.
#pragma once

#include <type_traits>

#include "sel_scan.cuh"

namespace snn {
namespace sscan {

constexpr int kSms = 152;

// Cuts for `warps` warps of a whole axis: as many as fit among the `resident` warps
// that the GPU holds at once.  Every cut costs each later warp a step at its start, so
// that a span is of kMinSpan tokens at least and no more than sqrt(3 T / 2) of them are worth it
// (400 tokens of 2048 channels, 16 states, bf16: 17 us forward and 38 backward, 24 and 58
// with spans of 64 tokens at least; 1024 tokens of 512 channels: 19 and 43, 24 and 51 without
// the root).  Below kMinCut tokens the axis stays whole: 100 tokens of 1024 channels take
// 15.0 us in one launch and 13.4 in spans, but a launch more.
constexpr int kMinSpan = 16, kMinCut = 128, kMaxSpans = 64;
// The kernel that finds their ends holds more warps.  Where its last round would stay
// empty it takes half spans (2 x 4096 tokens of 4096 channels: backward 720 us, 729 whole; 8 x
// 2048 tokens of 2048 775 and 820), but not below kMinHalf tokens (3 x 777 tokens of 1000 channels:
// 150 us of the training step, 144 whole) and never quarters (15 us in the second kernel).
constexpr int kEndsResident = kSms * 21, kMinHalf = 64;
inline double filled(int64_t warps, int64_t resident) {
  return warps > 0 ? (double)warps / (double)(ceil_div(warps, resident) * resident) : 0.0;
}
inline Plan cut(int64_t T, int64_t warps, int64_t resident) {
  int64_t most = T >= kMinCut ? T / kMinSpan : 1, spans = warps > 0 ? resident / warps : 1;
  if (most > kMaxSpans) most = kMaxSpans;
  while (most > 1 && 2 * most * most > 3 * T) --most;
  if (spans > most) spans = most;
  if (spans < 1) spans = 1;
  const bool halves = T / (2 * spans) >= kMinHalf && filled((spans - 1) * 2 * warps, kEndsResident) >
                                                         filled((spans - 1) * warps, kEndsResident) + 0.2;
  const int fine = halves ? 2 : 1;
  Plan p;
  p.fine = fine;
  p.span_fine = (int)round_up(T > 0 ? ceil_div(T, spans * fine) : 1, kTile);
  p.span = fine * p.span_fine;
  p.spans = T > 0 ? (int)ceil_div(T, p.span) : 1;
  return p;
}

// States of a thread and threads of a pair.  Backward of 2 x 4096 tokens of 4096 channels, 16
// states, as the kernel was when each was tried: eight states in two threads 553 us, four
// in four 882 (every operand from shared memory serves two channels of four
// states), sixteen in one 662 (255 registers, eight warps an SM).  17 to 24 states: twelve in
// two 95 us at 3 x 777 tokens of 1000 channels, eight in four 104.
struct Lay {
  int NS, P;
};
inline Lay lay_of(int N) {
  return N <= 4 ? Lay{4, 1} : N <= 8 ? Lay{4, 2} : N <= 16 ? Lay{8, 2} : N <= 24 ? Lay{12, 2}
       : N <= 32 ? Lay{8, 4} : N <= 48 ? Lay{12, 4} : Lay{16, 4};
}
inline int64_t warps_of(const Args& g, Lay l) { return (int64_t)g.B * g.G * ceil_div(g.pairs, 32 / l.P); }

// f(states, threads) as constants (kNarrow: of a forward pass, whose plan may take four
// threads for 9 to 16 states).
template <bool kNarrow, typename F>
cudaError_t with_lay(Lay l, F f) {
  using std::integral_constant;
  if (l.P == 1) return f(integral_constant<int, 4>(), integral_constant<int, 1>());
  if (l.P == 2) {
    if (l.NS == 4) return f(integral_constant<int, 4>(), integral_constant<int, 2>());
    if (l.NS == 8) return f(integral_constant<int, 8>(), integral_constant<int, 2>());
    return f(integral_constant<int, 12>(), integral_constant<int, 2>());
  }
  if constexpr (kNarrow)
    if (l.NS == 4) return f(integral_constant<int, 4>(), integral_constant<int, 4>());
  if (l.NS == 8) return f(integral_constant<int, 8>(), integral_constant<int, 4>());
  if (l.NS == 12) return f(integral_constant<int, 12>(), integral_constant<int, 4>());
  return f(integral_constant<int, 16>(), integral_constant<int, 4>());
}

struct FwdPlan {
  Lay lay;
  Plan cut;
};
inline FwdPlan fwd_plan(const Args& g) {
  FwdPlan p;
  p.lay = lay_of(g.N);
  // too few channels and tokens to fill the GPU: more threads to a pair (100 tokens of 1024
  // channels, 16 states: 15 us, 20 with two threads; 777 tokens of 1001 channels 35 and 64)
  const int64_t spans = g.T >= 64 ? g.T / 64 : 1;
  if (warps_of(g, p.lay) * spans < kSms * 8 && g.N > 8 && g.N <= 24)
    p.lay = g.N <= 16 ? Lay{4, 4} : Lay{8, 4};
  // the warps of an SM that their registers leave (2 x 1500 tokens of 1536 channels, 20
  // states: 64 us with 12, 79 with 16; 16 states, 2 x 4096 tokens of 4096 channels: 328 with 12, 319
  // with 16)
  p.cut = cut(g.T, warps_of(g, p.lay), kSms * (p.lay.NS <= 8 ? 16 : p.lay.NS == 12 ? 12 : 9));
  return p;
}
inline void put_cut(Args& g, const Plan& p) {
  g.spans = p.spans;
  g.span = p.span;
  g.fine = p.fine;
  g.span_fine = p.span_fine;
}
inline size_t fwd_bytes(const Args& g, const FwdPlan& p) {
  return p.cut.spans > 1 ? ends_bytes(g, p.cut.spans * p.cut.fine) + sums_bytes(g, p.cut.spans * p.cut.fine) : 0;
}

cudaError_t launch_back_ends(const Args& g, Lay lay, int dtype, cudaStream_t st);

}  // namespace sscan
}  // namespace snn
