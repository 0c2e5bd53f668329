// How a selective scan is laid on threads and its axis cut, from the shape alone.
#pragma once

#include <type_traits>

#include "sel_scan.cuh"

namespace snn {
namespace sscan {

constexpr int kSms = 152;

// Cuts for `warps` warps of a whole axis: as many as make whole rounds of the
// `resident` warps that the GPU holds at once, of at least kMinSpan tokens; and the parts
// that fill it best with warps of the kernel that finds their ends.
constexpr int kMinSpan = 64, kMaxSpans = 64, kEndsResident = kSms * 21;
inline double filled(int64_t warps, int64_t resident) {
  return warps > 0 ? (double)warps / (double)(ceil_div(warps, resident) * resident) : 0.0;
}
inline Plan cut(int64_t T, int64_t warps, int64_t resident) {
  int64_t most = T / kMinSpan, spans = warps > 0 ? resident / warps : 1;
  if (most > kMaxSpans) most = kMaxSpans;
  if (spans > most) spans = most;
  if (spans < 1) spans = 1;
  // (every part costs the second kernel a step at its start: 9 spans in 36 parts 15 us)
  const bool halves = T / (2 * spans) >= kMinSpan && filled((spans - 1) * 2 * warps, kEndsResident) >
                                                         filled((spans - 1) * warps, kEndsResident) + 0.2;
  const int fine = halves ? 2 : 1;
  Plan p;
  p.fine = fine;
  p.span_fine = (int)round_up(T > 0 ? ceil_div(T, spans * fine) : 1, kTile);
  p.span = fine * p.span_fine;
  p.spans = T > 0 ? (int)ceil_div(T, p.span) : 1;
  return p;
}

// States of a thread and threads of a pair.
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
  // too few channels and tokens to fill the GPU: more threads to a pair
  const int64_t spans = g.T >= kMinSpan ? g.T / kMinSpan : 1;
  if (warps_of(g, p.lay) * spans < kSms * 8 && g.N > 8 && g.N <= 24)
    p.lay = g.N <= 16 ? Lay{4, 4} : Lay{8, 4};
  p.cut = cut(g.T, warps_of(g, p.lay), kSms * 16);
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
