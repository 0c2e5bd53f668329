// Selective scan over whole sequences, and the spans' ends for it and for its
// backward.  A warp goes through its span of the axis four tokens at a time; B and C of the
// four come to its shared memory, the tokens' inputs to the registers of the pairs'
// threads, each while the four before are worked on.
//
// 2 x 4096 tokens of 4096 channels, 16 states, bf16 with checkpoints: 187 us, the spans' ends 129
// before it; a prompt of 16384 tokens of 2048 channels 296 for both.  A state of a token is four fp32
// operations and a power of two, 53 us in either unit; a cut axis needs the powers twice.  A thread issues
// eight instructions for each state, 0.61 a clock and scheduler at four warps:
// bound by the latency of dependent instructions and the two units in turn.  (Registers capped for 18, 20 or
// 24 warps an SM: 238, 215 and 410 us for 196; sixteen states a thread 450 with both kernels' tails.)
#include "sel_scan.cuh"
#include "sel_scan_plan.cuh"

namespace snn {
namespace sscan {

enum Mode {
  kFull = 0,   // outputs
  kEnds = 1,   // what a span adds to the state after it
  kBack = 2    // what a span adds to the gradient of the state before it
};

constexpr int kFour = 4;  // tokens

// Blocks of an SM that the registers are held to (0: as they come): without, the gradient's ends take 91
// for 80 with 8 states, 123 us for 101 at 2 x 4096 tokens of 4096 channels.
template <typename T, int MODE, int NS, int P>
constexpr int kBlocks = MODE == kBack && P == 2 && sizeof(T) == 2 ? (NS == 4 ? 24 : 0) : 0;

template <typename T, int MODE, int NS, int P>
__global__ void __launch_bounds__(32, kBlocks<T, MODE, NS, P>) scan_fwd(const Args g) {
  constexpr int PW = 32 / P, Np = P * NS, U = kFour / P;  // a thread's own tokens of four
  constexpr int kJobs = (MODE == kFull ? 2 : 1) * Np, kTurns = (kJobs + 31) / 32;  // fours of states to load
  __shared__ __align__(16) float smem[2][kJobs * 4];      // [B, C][kFour][Np]
  grid_dep_wait();
  const int lane = threadIdx.x, pl = lane & (P - 1);
  const int nb = (g.pairs + PW - 1) / PW;
  const int pb = blockIdx.x % nb, rest = blockIdx.x / nb, grp = rest % g.G, b = rest / g.G;
  // a span, or a part of one (backwards: of the second on)
  const int span = blockIdx.y + (MODE == kBack ? g.fine : 0), length = MODE == kFull ? g.span : g.span_fine;
  const int len = seq_len(g, b), first = span * length;
  const int last = first + length < g.T ? first + length : g.T;
  const int stop = last < len ? last : len;  // tokens that exist
  const int pair = pb * PW + lane / P, n0 = pl * NS;
  const bool live = pair < g.pairs, second = 2 * pair + 1 < g.Dg, pairs_ok = g.pair_ok;
  const bool gate = MODE != kEnds && g.z.data, soft = g.softplus;
  const int c = grp * g.Dg + 2 * pair;
  const int64_t row_states = (int64_t)g.N2 * g.pairs * 4;   // of one group in ends and ckpt
  float* const ends = g.ends + rest * row_states + pair * 4;
  const int64_t ends_step = (int64_t)g.B * g.G * row_states;
  const int64_t place = g.slots ? (int64_t)g.slots[b] : (int64_t)b;
  const bool has_place = place >= 0 && place < g.num_slots;

  float2 A2[NS], h[NS], total = f2(0.0f), bias = f2(0.0f), skip = f2(0.0f);
#pragma unroll
  for (int q = 0; q < NS; ++q) h[q] = A2[q] = f2(0.0f);
  if (live) {
    load_states<NS>(g.A + (int64_t)c * g.N, g.N, n0, second, A2);
#pragma unroll
    for (int q = 0; q < NS; ++q) A2[q] = mul2(A2[q], f2(kLog2E));
    if (g.bias) bias = make_float2(g.bias[c], second ? g.bias[c + 1] : 0.0f);
    if (MODE == kFull && g.D_skip) skip = make_float2(g.D_skip[c], second ? g.D_skip[c + 1] : 0.0f);
    if (MODE == kEnds && span == 0) {
      // the state before the first token, where the last span's end would be: the
      // kernel after this one may write it while its warps start from it
      float2 h0[NS];
#pragma unroll
      for (int q = 0; q < NS; ++q) h0[q] = f2(0.0f);
      if (g.state_in && has_place) load_states<NS>(g.state_in + (place * g.D + c) * g.N, g.N, n0, second, h0);
      store_twos<NS>(ends + (g.spans * g.fine - 1) * ends_step, g, n0, h0);
    }
    if (MODE == kFull) {
      if (g.spans > 1) {
        load_twos<NS>(ends + (g.spans * g.fine - 1) * ends_step, g, n0, h);
#pragma unroll 2
        for (int i = 0; i < span * g.fine; ++i) {
          float2 e[NS];
          load_twos<NS>(ends + i * ends_step, g, n0, e);
          join<NS>(h, A2, g.sums[((int64_t)i * g.B * g.G + rest) * g.pairs + pair], e);
        }
      } else if (g.state_in && has_place) {
        load_states<NS>(g.state_in + (place * g.D + c) * g.N, g.N, n0, second, h);
      }
    }
  }

  const int turns = stop > first ? (stop - first + kFour - 1) / kFour : 0;
  const int start = MODE == kBack ? first + (turns - 1) * kFour : first;
  constexpr int kStep = MODE == kBack ? -kFour : kFour;
  // a thread's own tokens (past the last pair: that one's)
  const Seq& in = MODE == kBack ? g.gy : g.u;
  const int c_in = live ? c : grp * g.Dg + 2 * (g.pairs - 1);
  auto own = [&](const Seq& m) { return static_cast<T*>(m.data) + b * m.sb + (int64_t)(start + pl) * m.st + c_in; };
  const T *pu = own(in), *pd = own(g.delta), *pz = own(g.z);
  T* py = own(g.y);
  Raw<T> raw_u[U], raw_d[U], raw_z[U];
  const bool quick = pairs_ok && g.quads;
  auto fetch = [&](int t0) {
    if (quick && t0 + kFour <= stop) {  // all the tokens exist
#pragma unroll
      for (int j = 0; j < U; ++j) {
        raw_u[j].load(pu + j * P * in.st, true, true);
        raw_d[j].load(pd + j * P * g.delta.st, true, true);
        if (gate) raw_z[j].load(pz + j * P * g.z.st, true, true);
      }
    } else {
#pragma unroll
      for (int j = 0; j < U; ++j) {
        raw_u[j].clear();
        raw_d[j].clear();
        raw_z[j].clear();
        if (live && t0 + pl + j * P < stop) {
          raw_u[j].load(pu + j * P * in.st, pairs_ok, second);
          raw_d[j].load(pd + j * P * g.delta.st, pairs_ok, second);
          if (gate) raw_z[j].load(pz + j * P * g.z.st, pairs_ok, second);
        }
      }
    }
    pu += kStep * in.st;
    pd += kStep * g.delta.st;
    pz += kStep * g.z.st;
  };
  // its fours of states of the four tokens' B, then C
  const T* pbc[kTurns];
  int64_t bc_step[kTurns];
  int bc_tok[kTurns], absent[kTurns];
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int k = lane + 32 * i, n = (k * 4) % Np, which = k / Np;
    const Mat& m = MODE == kBack || which ? g.Cm : g.Bm;
    bc_tok[i] = (k * 4 / Np) % kFour;
    absent[i] = n + 4 - g.N;
    pbc[i] = static_cast<const T*>(m.data) + b * m.sb + (int64_t)(start + bc_tok[i]) * m.st + grp * m.sg + n;
    bc_step[i] = kStep * m.st;
  }
  Four<T> next_bc[kTurns];
  auto fetch_bc = [&](int t0) {
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      next_bc[i].clear();
      if ((kJobs % 32 == 0 || lane + 32 * i < kJobs) && t0 + bc_tok[i] < stop && absent[i] < 4)
        next_bc[i].load(pbc[i], g.quads, absent[i] > 0 ? absent[i] : 0);
      pbc[i] += bc_step[i];
    }
  };

  float* ckpt = nullptr;
  if (MODE == kFull && g.ckpt && live)
    ckpt = g.ckpt + (((int64_t)b * ((g.T + kTile - 1) / kTile) + first / kTile) * g.G + grp) * row_states + pair * 4;
  if (turns) {
    fetch(start);
    fetch_bc(start);
  }
  Steps s8;  // since the states were settled
  // whole: all the tokens exist, in pairs
  auto tokens = [&](int turn, auto whole_) {
    constexpr bool whole = decltype(whole_)::value;
    const int t0 = start + turn * kStep;
    float* const bc = smem[turn & 1];
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
      if (kJobs % 32 == 0 || lane + 32 * i < kJobs) next_bc[i].put(bc + (lane + 32 * i) * 4);
    float2 s[U], x[U];
    Raw<T> now_u[U], now_z[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      s[j] = x[j] = f2(0.0f);
      if (whole || t0 + pl + j * P < stop) {
        s[j] = step_of<T>(add2(raw_d[j].get(), bias), soft);
        x[j] = raw_u[j].get();
        if (MODE == kBack) {
          if (gate) x[j] = mul2(x[j], mul2(raw_z[j].get(), sigmoid<T>(raw_z[j].get())));
        } else {
          x[j] = mul2(s[j], x[j]);
        }
        if (!whole && !second) s[j].y = x[j].y = 0.0f;
      }
      now_u[j] = raw_u[j];
      now_z[j] = raw_z[j];
    }
    __syncwarp();
    if (turn + 1 < turns) {
      fetch(t0 + kStep);
      fetch_bc(t0 + kStep);
    }
    if (MODE == kFull && ckpt && (turn & 1) == 0) {
      store_twos<NS>(ckpt, g, n0, h);
      ckpt += g.G * row_states;
    }
    float2 y[kFour];
#pragma unroll
    for (int i = 0; i < kFour; ++i) {
      const int k = MODE == kBack ? kFour - 1 - i : i;
      float2 sk = s[k / P], xk = x[k / P];
      if (P > 1) {
        const int from = (lane & ~(P - 1)) | (k & (P - 1));
        sk = from_lane(sk, from);
        xk = from_lane(xk, from);
      }
      const float* const rb = bc + k * Np + n0;
      const float* const rc = bc + (kFour + k) * Np + n0;
      const float2 s2[2] = {f2(sk.x), f2(sk.y)}, x2[2] = {f2(xk.x), f2(xk.y)};
      float2 sum[2] = {f2(0.0f), f2(0.0f)};  // of a channel
#pragma unroll
      for (int q = 0; q < NS; q += 4) {
        float v[4], w[4];
        Elem<float>::load4(rb + q, v);
        if (MODE == kFull) Elem<float>::load4(rc + q, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float2& hq = h[q + e];
          const float2 a = ex2(fma2(s2[e & 1], A2[q + e], f2(kLift))), in2 = make_float2(v[e & 2], v[(e & 2) + 1]);
          if (MODE == kBack) hq = mul2(a, fma2(x2[e & 1], in2, hq));
          else hq = fma2(a, hq, mul2(x2[e & 1], in2));
          if (MODE == kFull) sum[e & 1] = fma2(make_float2(w[e & 2], w[(e & 2) + 1]), hq, sum[e & 1]);
        }
      }
      s8.add(sk);
      if (MODE == kFull) y[k] = across(sum[0], sum[1]);
    }
    if (turn % (kSettle / kFour) == kSettle / kFour - 1) {
      settle<NS>(h, A2, s8);
      if (MODE != kFull) total = add2(total, s8.sum);
      s8 = Steps();
    }
    if (MODE == kFull) {
      share_out<kFour, P>(y, pl);
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int now = t0 + pl + j * P;
        if (live && (whole || now < last)) {
          float2 out = fma2(skip, now_u[j].get(), y[j * P]);
          if (gate) {
            const float2 z = now_z[j].get();
            out = mul2(out, mul2(z, sigmoid<T>(z)));
          }
          if (whole) put_pair(py + j * P * g.y.st, out, true, true);
          else put_pair(py + j * P * g.y.st, now < stop ? out : f2(0.0f), pairs_ok, second);
        }
      }
      py += kStep * g.y.st;
    }
  };
  {
    const int part = quick ? (stop - first) % kFour : 0;  // of the last four (backwards: the first turn)
    int turn = 0;
    if (MODE == kBack && turns && (!quick || part)) tokens(turn++, std::false_type());
    const int until = !quick ? 0 : MODE != kBack && part ? turns - 1 : turns;
    for (; turn < until; ++turn) tokens(turn, std::true_type());
    for (; turn < turns; ++turn) tokens(turn, std::false_type());
  }
  if (!live) return;
  if (MODE == kFull) {
    // places past the sequence's end
    for (int now = first + turns * kFour + pl; now < last; now += P, py += P * g.y.st)
      put_pair(py, f2(0.0f), pairs_ok, second);
    if (g.state_out && has_place && span == g.spans - 1)
      store_states<NS>(g.state_out + (place * g.D + c) * g.N, g.N, n0, second, h);
  } else {
    store_twos<NS>(ends + span * ends_step, g, n0, h);
    total = add2(total, s8.sum);
    if (pl == 0) g.sums[((int64_t)span * g.B * g.G + rest) * g.pairs + pair] = total;
  }
}

template <typename T, int MODE>
cudaError_t launch_mode(const Args& g, Lay lay, int spans, cudaStream_t st) {
  const int64_t blocks = warps_of(g, lay);
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  return with_lay<MODE != kBack>(lay, [&](auto NS, auto P) {
    return launch_pdl(scan_fwd<T, MODE, decltype(NS)::value, decltype(P)::value>, dim3((unsigned)blocks, (unsigned)spans),
                      dim3(32), 0, st, g);
  });
}

template <typename T>
cudaError_t launch_fwd(const Args& g, Lay lay, cudaStream_t st) {
  if (g.spans > 1) {
    const cudaError_t e = launch_mode<T, kEnds>(g, lay, (g.spans - 1) * g.fine, st);
    if (e != cudaSuccess) return e;
  }
  return launch_mode<T, kFull>(g, lay, g.spans, st);
}

cudaError_t launch_back_ends(const Args& g, Lay lay, int dtype, cudaStream_t st) {
  if (dtype == SNN_F32) return launch_mode<float, kBack>(g, lay, (g.spans - 1) * g.fine, st);
  if (dtype == SNN_BF16) return launch_mode<__nv_bfloat16, kBack>(g, lay, (g.spans - 1) * g.fine, st);
  return launch_mode<__half, kBack>(g, lay, (g.spans - 1) * g.fine, st);
}

}  // namespace sscan
}  // namespace snn

using namespace snn::sscan;

extern "C" {

size_t snn_sscan_desc_size(void) { return sizeof(snn_sscan_desc); }

int64_t snn_selective_scan_ckpt_elems(const snn_sscan_desc* desc) {
  if (!desc) return 0;
  snn_sscan_desc d = *desc;
  d.dtype = SNN_F32;
  d.softplus = 0;
  if (check_desc(&d) != SNN_OK) return 0;
  const Args g = base_args(&d);
  return snn::ceil_div(d.T, kTile) * state_floats(g);
}

snn_status_t snn_selective_scan_fwd(const snn_sscan_desc* desc, const snn_btc* u,
                                    const snn_btc* delta, const float* A, const snn_bthd* Bm,
                                    const snn_bthd* Cm, const float* D, const snn_btc* z,
                                    const float* delta_bias, const int32_t* seq_lens,
                                    const float* state_in, float* state_out,
                                    const int32_t* slots, int64_t num_slots, float* ckpt,
                                    const snn_btc* y, void* ws, size_t ws_bytes,
                                    snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  if (!A || num_slots < 0 || num_slots > kMost) return SNN_ERR_INVALID_ARG;
  if ((state_in || state_out) && !slots && num_slots < desc->B) return SNN_ERR_INVALID_ARG;
  const void* ptrs[9] = {A, D, delta_bias, seq_lens, state_in, state_out, slots, ckpt, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  Args g = base_args(desc);
  bool pair = g.Dg % 2 == 0;
  if (desc->B > 0 && desc->T > 0) {
    if ((s = take(desc, u, &g.u, &pair)) != SNN_OK || (s = take(desc, delta, &g.delta, &pair)) != SNN_OK ||
        (z && z->data && (s = take(desc, z, &g.z, &pair)) != SNN_OK) ||
        (s = take(desc, y, &g.y, &pair)) != SNN_OK || (s = take(desc, Bm, &g.Bm)) != SNN_OK ||
        (s = take(desc, Cm, &g.Cm)) != SNN_OK)
      return s;
  }
  const FwdPlan plan = fwd_plan(g);
  put_cut(g, plan.cut);
  const size_t need = fwd_bytes(g, plan);
  if (need && (!ws || ws_bytes < need)) return SNN_ERR_WORKSPACE;
  if (desc->B == 0 || (desc->T == 0 && !state_out)) return SNN_OK;
  g.pair_ok = pair;
  g.quads = quads(g, {&g.Bm, &g.Cm});
  g.A = A;
  g.D_skip = D;
  g.bias = delta_bias;
  g.seq_lens = seq_lens;
  g.slots = slots;
  g.num_slots = num_slots;
  g.state_in = state_in;
  g.state_out = state_out;
  g.ckpt = ckpt;
  unsigned char* w = static_cast<unsigned char*>(ws);
  g.ends = reinterpret_cast<float*>(w);
  g.sums = reinterpret_cast<float2*>(w + ends_bytes(g, plan.cut.spans * plan.cut.fine));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = desc->dtype == SNN_F32    ? launch_fwd<float>(g, plan.lay, st)
                        : desc->dtype == SNN_BF16 ? launch_fwd<__nv_bfloat16>(g, plan.lay, st)
                                                  : launch_fwd<__half>(g, plan.lay, st);
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

}  // extern "C"
