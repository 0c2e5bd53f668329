// Selective scan, backward.  With dy = grad_y silu(z) (the gradient of the sum over states
// and of D u), and gamma the gradient that reaches h_t from later tokens:
//   gt = dy C_t + gamma;        gamma <- a_t gt
//   grad_C = sum over channels of dy h_t;      grad_B = sum over channels of gt x
//   w = sum_n gt B;  q = a_t gt h_{t-1};  r = sum_n q A
//   grad_u = s w + D dy;   grad_delta = (u w + r) softplus'(delta + bias)
//   grad_A = sum_t q s;    grad_D = sum_t dy u;   grad_z = grad_y (y before the gate) silu'(z)
// A warp goes backwards through its span of the axis in tiles of the checkpoints' eight
// tokens: from the checkpoint it takes the states forwards through the tile and leaves them
// in tensor memory, which serves here as a second register file (sixteen words a
// token of a thread's lane; through shared memory they would be the bound), then
// gamma back through it.  grad_B and grad_C are summed over the warp's channels as the
// tokens pass, halving the values a thread holds with every exchange; the warps' shares, and
// those of grad_A, grad_D and grad_delta_bias, are added by further kernels in a fixed order.
//
// 2 x 4096 tokens of 4096 channels, 16 states, bf16: 552 us, the gradient's ends of the spans
// 140 before it, the sums 25 and 6 after it.  The formulas are 15 operations and two
// powers of two a state, 200 us at the rate of fp32; a thread issues 24 instructions for each
// state, 0.59 a clock and scheduler, and what keeps it there is the latency of dependent
// instructions at three warps a scheduler (168 registers; a fourth warp at 128: 661 us, the token loops
// unrolled by two: 640).  Tiles of a whole block between barriers took 2752, warps that
// work alone with four states to a thread and the sums through shared memory 879, eight states
// and tensor memory 696, inputs by asynchronous copies 620, whole tiles without checks 553.
#include "sel_scan.cuh"
#include "sel_scan_plan.cuh"
#include "tcgen05.cuh"

namespace snn {
namespace sscan {

using gemm::tc_fence_after;
using gemm::tc_fence_before;
using gemm::tmem_alloc;
using gemm::tmem_dealloc;

constexpr int kWarps = 4;        // of a block, one for each quarter of tensor memory
constexpr int kSettleTiles = kSettle / kTile;

struct BwdPlan {
  Lay lay;
  int blocks;  // warps of a group
  Plan cut;
};

// Columns of tensor memory: a tile's states, allocated in powers of two.
__host__ __device__ constexpr int columns_of(int NS) { return NS == 4 ? 64 : NS == 8 ? 128 : 256; }
// Blocks of an SM: 168 registers a thread, 255 for 12 and 16 states.
__host__ __device__ constexpr int blocks_of(int NS) { return NS <= 8 ? 3 : 2; }

BwdPlan bwd_plan(const Args& g) {
  BwdPlan p;
  p.lay = lay_of(g.N);
  p.blocks = (int)ceil_div(g.pairs, 32 / p.lay.P);
  p.cut = cut(g.T, warps_of(g, p.lay), kSms * kWarps * blocks_of(p.lay.NS));
  return p;
}

// Values of a sum over the warp's pairs, padded to a power of two.
__host__ __device__ constexpr int sums_of(int NS) { return NS == 12 ? 16 : NS; }
// Orders of a four of states (see order_of): whole numbers below this are xor-ed on it.
__host__ __device__ constexpr int copies_of(int NS, int P) { return NS == 12 ? 1 : NS * P / 32 > 1 ? 2 : 4; }
// Where order x lies: each in banks of its own.
__host__ __device__ constexpr int copy_at(int NS, int P, int x) { return x * kTile * 2 * P * NS + (x & 1) * 16 + (x >> 1) * 36; }

// Shared memory of a warp, in bytes.
template <typename T, int NS, int P>
struct Smem {
  static constexpr int PW = 32 / P, Np = P * NS;
  static constexpr int su = 0;                                                  // float4 [kTile][PW]: s, u
  static constexpr int sg = su + kTile * PW * 16;                               // float4 [kTile][PW]: softplus', grad_y silu'
  static constexpr int dy = sg + kTile * PW * 16;                               // float2 [kTile][PW]
  static constexpr int bc = dy + kTile * PW * 8;                                // [copies][kTile][B, C][Np]
  static constexpr int raw = bc + (copy_at(NS, P, copies_of(NS, P)) + 16) * 4;    // Raw [u, delta, grad_y, z][kTile][PW]
  static constexpr int raw_bc = raw + 4 * kTile * PW * (int)sizeof(Raw<T>);     // T [kTile][B, C][Np]
  static constexpr int h0 = raw_bc + 2 * kTile * Np * (int)sizeof(T);           // float4 [NS / 2][32]
  static constexpr int steps = h0 + NS / 2 * 32 * 16;                           // Steps [32]: of a thread's own tokens
  static constexpr int bytes = steps + 32 * 16;
};

// To shared memory without passing registers; there after copies_arrived().
template <int bytes>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  if constexpr (bytes == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(to)), "l"(from), "n"(bytes) : "memory");
}
__device__ __forceinline__ void copies_arrived() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Tensor memory as a thread's own: columns of its lane.  What is loaded is there after
// arrived().
__device__ __forceinline__ void own_load(uint32_t at, float2* v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(v[0].x), "=f"(v[0].y), "=f"(v[1].x), "=f"(v[1].y), "=f"(v[2].x), "=f"(v[2].y), "=f"(v[3].x),
                 "=f"(v[3].y)
               : "r"(at));
}
template <int NS>
__device__ __forceinline__ void arrived(float2 (&v)[NS]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;");
#pragma unroll
  for (int q = 0; q < NS; ++q) asm volatile("" : "+f"(v[q].x), "+f"(v[q].y));
}
__device__ __forceinline__ void own_store(uint32_t at, const float2* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"f"(v[0].x),
               "f"(v[0].y), "f"(v[1].x), "f"(v[1].y), "f"(v[2].x), "f"(v[2].y), "f"(v[3].x), "f"(v[3].y), "r"(at));
}
__device__ __forceinline__ void stored() { asm volatile("tcgen05.wait::st.sync.aligned;"); }

// Sums of K values (a power of two) over a warp's pairs, whose threads are P apart.  With
// each exchange a thread keeps half of the values; left are the first max(1, K P / 32).  Ordered: a
// thread's v[i] is value i ^ order_of(lane), so that what it keeps always comes first and nothing
// has to be selected.
template <int K, int P, bool kOrdered>
__device__ __forceinline__ void sum_over_pairs(float (&v)[K], int lane) {
#pragma unroll
  for (int o = 16; o >= P; o >>= 1) {
    const int n = K * o / 32;  // left after this exchange
    const bool up = lane & o;
    if (n >= 1) {
#pragma unroll
      for (int i = 0; i < n; ++i) {
        if (kOrdered) {
          v[i] += __shfl_xor_sync(0xffffffffu, v[i + n], o);
        } else {
          const float give = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
      }
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    }
  }
}
// The first value that is left, and whether another thread has the same ones.
template <int K, int P>
__device__ __forceinline__ int left_at(int lane, bool* twice) {
  int at = 0;
  *twice = false;
#pragma unroll
  for (int o = 16; o >= P; o >>= 1) {
    const int n = K * o / 32;
    if (lane & o) {
      if (n < 1) *twice = true;
      at += n;
    }
  }
  return at;
}
// State i <- state i ^ order.
template <int NS>
__device__ __forceinline__ void reorder(float2 (&v)[NS], int order) {
#pragma unroll
  for (int i = 0; i < NS; ++i) v[i] = order & 1 ? make_float2(v[i].y, v[i].x) : v[i];
#pragma unroll
  for (int n = 2; n < NS; n <<= 1) {
    const bool up = order & n;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      if (!(i & n)) {
        const float2 a = v[i], b = v[i ^ n];
        v[i] = up ? b : a;
        v[i ^ n] = up ? a : b;
      }
    }
  }
}

// A channel's value times a pair of states (plus c): as two instructions where four
// threads' turns leave no registers for the value twice.
template <bool kTwice>
__device__ __forceinline__ float2 times(float a, float2 v) {
  if constexpr (kTwice) return mul2(f2(a), v);
  else return make_float2(a * v.x, a * v.y);
}
template <bool kTwice>
__device__ __forceinline__ float2 times(float a, float2 v, float2 c) {
  if constexpr (kTwice) return fma2(f2(a), v, c);
  else return make_float2(fmaf(a, v.x, c.x), fmaf(a, v.y, c.y));
}

template <typename T, int NS, int P>
__device__ void scan_back(const Args& g, int64_t work, unsigned char* smem, uint32_t t_h) {
  using S = Smem<T, NS, P>;
  constexpr int K = sums_of(NS), kLeft = K * P / 32 > 1 ? K * P / 32 : 1;   // sums over pairs
  constexpr bool kOrdered = NS != 12, kTwice = P < 4;
  constexpr int kCopies = copies_of(NS, P);
  constexpr int PW = 32 / P, Np = P * NS, U = kTile / P;
  constexpr int kTokens = 128 / Np, kTurns = (kTile + kTokens - 1) / kTokens;  // whose B and C are loaded at once
  const int lane = threadIdx.x & 31, pl = lane & (P - 1), pc = lane / P;
  float4* const psu = reinterpret_cast<float4*>(smem + S::su) + pc;
  float4* const psg = reinterpret_cast<float4*>(smem + S::sg) + pc;
  float2* const pdy = reinterpret_cast<float2*>(smem + S::dy) + pc;
  float* const bc = reinterpret_cast<float*>(smem + S::bc);
  Raw<T>* const raw = reinterpret_cast<Raw<T>*>(smem + S::raw) + pc;
  T* const raw_bc = reinterpret_cast<T*>(smem + S::raw_bc);
  float4* const h0 = reinterpret_cast<float4*>(smem + S::h0) + lane;
  Steps* const steps = reinterpret_cast<Steps*>(smem + S::steps);

  const int nb = (g.pairs + PW - 1) / PW;
  const int64_t place = work / g.spans;
  const int span = (int)(work - place * g.spans);
  const int pb = (int)(place % nb), rest = (int)(place / nb), grp = rest % g.G, b = rest / g.G;
  const int len = seq_len(g, b), first = span * g.span;
  const int last = first + g.span < g.T ? first + g.span : g.T;
  const int stop = last < len ? last : len;
  const int tiles = stop > first ? (stop - first + kTile - 1) / kTile : 0;
  const int pair = pb * PW + pc, n0 = pl * NS;
  const bool live = pair < g.pairs, second = 2 * pair + 1 < g.Dg, pairs_ok = g.pair_ok, quads_ok = g.quads;
  const bool gate = g.z.data != nullptr, soft = g.softplus;
  const int c = grp * g.Dg + 2 * pair;
  const int64_t row_states = (int64_t)g.N2 * g.pairs * 4;
  // its shares of grad_B and grad_C, and the order of its states
  bool twice;
  const int at = left_at<K, P>(lane, &twice), order = kOrdered ? at : 0;
  const bool puts = !twice && at < NS && n0 + at < g.N;

  float2 A2[NS], gam[NS], dA[NS], bias = f2(0.0f), skip = f2(0.0f), sum_D = f2(0.0f), sum_bias = f2(0.0f);
#pragma unroll
  for (int q = 0; q < NS; ++q) A2[q] = gam[q] = dA[q] = f2(0.0f);
  if (live) {
    load_states<NS>(g.A + (int64_t)c * g.N, g.N, n0, second, A2);
#pragma unroll
    for (int q = 0; q < NS; ++q) A2[q] = mul2(A2[q], f2(kLog2E));
    if (g.bias) bias = make_float2(g.bias[c], second ? g.bias[c + 1] : 0.0f);
    if (g.D_skip) skip = make_float2(g.D_skip[c], second ? g.D_skip[c + 1] : 0.0f);
    if (g.grad_state_out) load_states<NS>(g.grad_state_out + ((int64_t)b * g.D + c) * g.N, g.N, n0, second, gam);
    for (int i = g.spans * g.fine - 1; i >= (span + 1) * g.fine; --i) {
      float2 e[NS];
      load_twos<NS>(g.ends + ((int64_t)i * g.B * g.G + rest) * row_states + pair * 4, g, n0, e);
      join<NS>(gam, A2, g.sums[((int64_t)i * g.B * g.G + rest) * g.pairs + pair], e);
    }
  }
  if (kOrdered) {
    reorder<NS>(A2, order);
    reorder<NS>(gam, order);
  }

  // a thread's own tokens of the last tile, and its fours of states of B and C
  const int t_last = first + (tiles - 1) * kTile;
  // (past the last pair: that one's inputs, with s and dy of zero)
  const int pair_in = live ? pair : g.pairs - 1;
  auto own = [&](const Seq& m) {
    return static_cast<T*>(m.data) + b * m.sb + (int64_t)(t_last + pl) * m.st + grp * g.Dg + 2 * pair_in;
  };
  const T *in_u = own(g.u), *in_d = own(g.delta), *in_g = own(g.gy), *in_z = own(g.z);
  T *out_u = own(g.gu), *out_d = own(g.gdelta), *out_z = own(g.gz);
  const float* ckpt = g.ckpt + (((int64_t)b * ((g.T + kTile - 1) / kTile) + t_last / kTile) * g.G + grp) * row_states +
                      ((int64_t)(n0 / 2) * g.pairs + pair_in) * 4;
  const int bc_tok = lane * 4 / Np, bc_n = lane * 4 % Np, absent = bc_n + 4 - g.N > 0 ? bc_n + 4 - g.N : 0;
  const T* pB = static_cast<const T*>(g.Bm.data) + b * g.Bm.sb + (int64_t)(t_last + bc_tok) * g.Bm.st + grp * g.Bm.sg + bc_n;
  const T* pC = static_cast<const T*>(g.Cm.data) + b * g.Cm.sb + (int64_t)(t_last + bc_tok) * g.Cm.st + grp * g.Cm.sg + bc_n;
  const int64_t part_step = (int64_t)g.G * g.N;
  const int64_t part0 = ((((int64_t)pb * g.B + b) * g.T + t_last) * g.G + grp) * g.N + n0 + at;
  float *part_B = g.part_B + part0 + (kTile - 1) * part_step, *part_C = g.part_C + part0;
  auto put_part = [&](float* p, const float (&v)[K]) {
#pragma unroll
    for (int j = 0; j < kLeft; ++j)
      if (j == 0 || n0 + at + j < g.N) p[j] = v[j];
  };

  // a tile's inputs on their way to shared memory; quick: all of them, in whole vectors
  const bool quick = pairs_ok && quads_ok;
  auto fetch = [&](int tokens) {
    if (quick && tokens == kTile) {
#pragma unroll
      for (int j = 0; j < U; ++j) {
        Raw<T>* const to = raw + (pl + j * P) * PW;
        copy_async<sizeof(Raw<T>)>(to, in_u + j * P * g.u.st);
        copy_async<sizeof(Raw<T>)>(to + kTile * PW, in_d + j * P * g.delta.st);
        copy_async<sizeof(Raw<T>)>(to + 2 * kTile * PW, in_g + j * P * g.gy.st);
        if (gate) copy_async<sizeof(Raw<T>)>(to + 3 * kTile * PW, in_z + j * P * g.z.st);
      }
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int tok = bc_tok + i * kTokens;
        if (tok < kTile && bc_tok < kTokens && absent == 0) {
          copy_async<4 * sizeof(T)>(raw_bc + tok * 2 * Np + bc_n, pB + i * kTokens * g.Bm.st);
          copy_async<4 * sizeof(T)>(raw_bc + (tok * 2 + 1) * Np + bc_n, pC + i * kTokens * g.Cm.st);
        }
      }
#pragma unroll
      for (int k = 0; k < NS / 2; ++k)
        if (n0 / 2 + k < g.N2) copy_async<16>(h0 + k * 32, ckpt + (int64_t)k * g.pairs * 4);
    } else {
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int tok = pl + j * P;
        Raw<T>* const to = raw + tok * PW;
        auto one = [&](int k, const T* p) {
          Raw<T> r;
          r.clear();
          if (live && tok < tokens) r.load(p, pairs_ok, second);
          to[k * kTile * PW] = r;
        };
        one(0, in_u + j * P * g.u.st);
        one(1, in_d + j * P * g.delta.st);
        one(2, in_g + j * P * g.gy.st);
        if (gate) one(3, in_z + j * P * g.z.st);
      }
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int tok = bc_tok + i * kTokens;
        if (tok < kTile && bc_tok < kTokens) {
          auto one = [&](int k, const T* p) {
            Four<T> r;
            r.clear();
            if (tok < tokens && absent < 4) r.load(p, quads_ok, absent);
            *reinterpret_cast<Four<T>*>(raw_bc + (tok * 2 + k) * Np + bc_n) = r;
          };
          one(0, pB + i * kTokens * g.Bm.st);
          one(1, pC + i * kTokens * g.Cm.st);
        }
      }
#pragma unroll
      for (int k = 0; k < NS / 2; ++k) {
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (live && n0 / 2 + k < g.N2) v = *reinterpret_cast<const float4*>(ckpt + (int64_t)k * g.pairs * 4);
        h0[k * 32] = v;
      }
    }
    in_u -= kTile * g.u.st;
    in_d -= kTile * g.delta.st;
    in_g -= kTile * g.gy.st;
    in_z -= kTile * g.z.st;
    pB -= kTile * g.Bm.st;
    pC -= kTile * g.Cm.st;
    ckpt -= g.G * row_states;
  };
  auto tokens_of = [&](int tile) {
    const int n = stop - (first + tile * kTile);
    return n < kTile ? n : kTile;
  };
  {  // absent states stay zero
#pragma unroll
    for (int k = 0; k < NS / 2; ++k)
      if (n0 / 2 + k >= g.N2) h0[k * 32] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const int tok = bc_tok + i * kTokens;
      if (tok < kTile && bc_tok < kTokens && absent > 0) {
        Four<T> r;
        r.clear();
        *reinterpret_cast<Four<T>*>(raw_bc + tok * 2 * Np + bc_n) = r;
        *reinterpret_cast<Four<T>*>(raw_bc + (tok * 2 + 1) * Np + bc_n) = r;
      }
    }
  }
  if (tiles) fetch(tokens_of(tiles - 1));
  const float* const bc_own = bc + copy_at(NS, P, kCopies == 1 ? 0 : kCopies == 2 ? (order >> 1) & 1 : order & 3) + n0;
  const int first_four = order >> 2;

  // gamma, after kSettleTiles tiles: of 16-bit inputs at the end of the last of them, of 32-bit ones
  // at the start of the next (2 x 4096 tokens of 4096 channels, 16 states: fp32 807 us, 825 at the end; bf16 of 24 states
  // 575 at the end and 589)
  auto settle_all = [&]() {
    Steps all;
#pragma unroll
    for (int k = 0; k < P; ++k) all.add(steps[(lane & ~(P - 1)) + k]);
    settle<NS>(gam, A2, all);
  };
  for (int tile = tiles - 1; tile >= 0; --tile) {
    const int tokens = tokens_of(tile);
    copies_arrived();
    __syncwarp();
    if (sizeof(T) == 4 && tile != tiles - 1 && tile % kSettleTiles == kSettleTiles - 1) {
      settle_all();
      __syncwarp();
    }
    float2 h[NS];
#pragma unroll
    for (int k = 0; k < NS / 2; ++k) {
      const float4 v = h0[(kOrdered ? k ^ (order >> 1) : k) * 32];
      const bool swap = kOrdered && (order & 1);
      h[2 * k] = swap ? make_float2(v.y, v.x) : make_float2(v.x, v.y);
      h[2 * k + 1] = swap ? make_float2(v.w, v.z) : make_float2(v.z, v.w);
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const int tok = bc_tok + i * kTokens;
      if (tok < kTile && bc_tok < kTokens) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float v[4];
          reinterpret_cast<const Four<T>*>(raw_bc + (tok * 2 + k) * Np + bc_n)->put(v);
          float* const to = bc + (tok * 2 + k) * Np + bc_n;
#pragma unroll
          for (int x = 0; x < kCopies; ++x) {
            const int y = kCopies == 2 ? 2 * x : x;
            *reinterpret_cast<float4*>(to + copy_at(NS, P, x)) = make_float4(v[y], v[1 ^ y], v[2 ^ y], v[3 ^ y]);
          }
        }
      }
    }
    Steps own_steps;
    if (tile % kSettleTiles != kSettleTiles - 1 && tile != tiles - 1) own_steps = steps[lane];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int tok = pl + j * P;
      const Raw<T>* const from = raw + tok * PW;
      const float2 u = from[0].get();
      float2 s = f2(0.0f), dy = from[2 * kTile * PW].get(), slope = f2(0.0f), gz = f2(0.0f);
      if (quick && tokens == kTile) s = step_of<T>(add2(from[kTile * PW].get(), bias), soft, &slope);
      else if (live && tok < tokens) s = step_of<T>(add2(from[kTile * PW].get(), bias), soft, &slope);
      if (gate) {
        const float2 z = from[3 * kTile * PW].get(), sig = sigmoid<T>(z), zs = mul2(z, sig);
        gz = mul2(dy, fma2(zs, fma2(sig, f2(-1.0f), f2(1.0f)), sig));
        dy = mul2(dy, zs);
      }
      if (!live) s = dy = f2(0.0f);
      if (!second) s.y = dy.y = 0.0f;
      own_steps.add(s);
      psu[tok * PW] = make_float4(s.x, s.y, u.x, u.y);
      psg[tok * PW] = make_float4(slope.x, slope.y, gz.x, gz.y);
      pdy[tok * PW] = dy;
    }
    steps[lane] = own_steps;
    __syncwarp();
    if (tile > 0) fetch(kTile);
    // the states forwards
#pragma unroll 1
    for (int i0 = 0; i0 < kTile; i0 += P) {
      float2 y[P];
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const int i = i0 + k;
#pragma unroll
        for (int q = 0; q < NS; q += 4) own_store(t_h + i * 2 * NS + 2 * q, h + q);
        const float4 su = psu[i * PW];
        const float2 s = make_float2(su.x, su.y), x = mul2(s, make_float2(su.z, su.w)), dy = pdy[i * PW];
        const float sj[2] = {s.x, s.y}, xj[2] = {x.x, x.y}, dyj[2] = {dy.x, dy.y};
        const float* const rb = bc_own + i * 2 * Np;
        float2 sum[2] = {f2(0.0f), f2(0.0f)};
        float dC[K];
#pragma unroll
        for (int q = 0; q < NS; q += 4) {
          float v[4], w[4];
          const int four = kOrdered ? 4 * ((q / 4) ^ first_four) : q;
          Elem<float>::load4(rb + four, v);
          Elem<float>::load4(rb + Np + four, w);
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const float2 v2 = make_float2(v[e], v[e + 1]), w2 = make_float2(w[e], w[e + 1]);
            float2 *const hq = h + q + e, d = f2(0.0f);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              hq[j] = fma2(ex2(times<kTwice>(sj[j], A2[q + e + j], f2(kLift))), hq[j], times<kTwice>(xj[j], v2));
              sum[j] = fma2(w2, hq[j], sum[j]);
              d = j ? times<kTwice>(dyj[j], hq[j], d) : times<kTwice>(dyj[j], hq[j]);
            }
            dC[q + e] = d.x;
            dC[q + e + 1] = d.y;
          }
        }
        y[k] = across(sum[0], sum[1]);
#pragma unroll
        for (int q = NS; q < K; ++q) dC[q] = 0.0f;
        sum_over_pairs<K, P, kOrdered>(dC, lane);
        if (puts && i < tokens) put_part(part_C, dC);
        part_C += part_step;
      }
      if (gate) {
        share_out<P, P>(y, pl);
        const int i = i0 + pl;
        if (live && i < tokens) {
          const float4 su = psu[i * PW], sg = psg[i * PW];
          put_pair(out_z + i0 * g.gz.st,
                   mul2(make_float2(sg.z, sg.w), fma2(skip, make_float2(su.z, su.w), y[0])), pairs_ok, second);
        }
      }
    }
    stored();
    // gamma backwards
#pragma unroll 1
    for (int i0 = kTile - P; i0 >= 0; i0 -= P) {
      float2 w[P], r[P];
#pragma unroll
      for (int k = P - 1; k >= 0; --k) {
        const int i = i0 + k;
        float2 hv[NS];
#pragma unroll
        for (int q = 0; q < NS; q += 4) own_load(t_h + i * 2 * NS + 2 * q, hv + q);
        const float4 su = psu[i * PW];
        const float2 s = make_float2(su.x, su.y), x = mul2(s, make_float2(su.z, su.w)), dy = pdy[i * PW];
        const float sj[2] = {s.x, s.y}, xj[2] = {x.x, x.y}, dyj[2] = {dy.x, dy.y};
        const float* const rb = bc_own + i * 2 * Np;
        float2 sw[2] = {f2(0.0f), f2(0.0f)}, sr[2] = {f2(0.0f), f2(0.0f)};
        float dB[K];
#pragma unroll
        for (int q = 0; q < NS; q += 4) {
          float vb[4], vc[4];
          const int four = kOrdered ? 4 * ((q / 4) ^ first_four) : q;
          Elem<float>::load4(rb + four, vb);
          Elem<float>::load4(rb + Np + four, vc);
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const float2 b2 = make_float2(vb[e], vb[e + 1]), c2 = make_float2(vc[e], vc[e + 1]);
            float2 *const gq = gam + q + e, d = f2(0.0f);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              gq[j] = times<kTwice>(dyj[j], c2, gq[j]);
              d = j ? times<kTwice>(xj[j], gq[j], d) : times<kTwice>(xj[j], gq[j]);
              sw[j] = fma2(b2, gq[j], sw[j]);
              gq[j] = mul2(ex2(times<kTwice>(sj[j], A2[q + e + j], f2(kLift))), gq[j]);
            }
            dB[q + e] = d.x;
            dB[q + e + 1] = d.y;
          }
        }
        arrived<NS>(hv);
#pragma unroll
        for (int q = 0; q < NS; ++q) {
          const float2 qq = mul2(gam[q], hv[q]);
          sr[q & 1] = fma2(qq, A2[q], sr[q & 1]);
          dA[q] = times<kTwice>(sj[q & 1], qq, dA[q]);
        }
        w[k] = across(sw[0], sw[1]);
        r[k] = across(sr[0], sr[1]);
#pragma unroll
        for (int q = NS; q < K; ++q) dB[q] = 0.0f;
        sum_over_pairs<K, P, kOrdered>(dB, lane);
        if (puts && i < tokens) put_part(part_B, dB);
        part_B -= part_step;
      }
      share_out<P, P>(w, pl);
      share_out<P, P>(r, pl);
      const int i = i0 + pl;
      if (live && i < tokens) {
        const float4 su = psu[i * PW], sg = psg[i * PW];
        const float2 s = make_float2(su.x, su.y), u = make_float2(su.z, su.w), dy = pdy[i * PW];
        const float2 du = fma2(s, w[0], mul2(skip, dy));
        // r holds A log2(e)
        const float2 dd = mul2(fma2(u, w[0], mul2(r[0], f2(0.69314718055994530942f))), make_float2(sg.x, sg.y));
        put_pair(out_u + i0 * g.gu.st, du, pairs_ok, second);
        put_pair(out_d + i0 * g.gdelta.st, dd, pairs_ok, second);
        sum_D = fma2(dy, u, sum_D);
        sum_bias = add2(sum_bias, dd);
      }
    }
    if (sizeof(T) == 2 && tile % kSettleTiles == 0) settle_all();
    out_u -= kTile * g.gu.st;
    out_d -= kTile * g.gdelta.st;
    out_z -= kTile * g.gz.st;
    part_C -= 2 * kTile * part_step;
    __syncwarp();
  }

  sum_D = sum_pair<P>(sum_D);
  sum_bias = sum_pair<P>(sum_bias);
  if (!live) return;
  // places past the sequence's end
  auto base = [&](const Seq& x, int now) { return static_cast<T*>(x.data) + b * x.sb + now * x.st + c; };
  for (int now = (stop > first ? stop : first) + pl; now < last; now += P) {
    put_pair(base(g.gu, now), f2(0.0f), pairs_ok, second);
    put_pair(base(g.gdelta, now), f2(0.0f), pairs_ok, second);
    if (gate) put_pair(base(g.gz, now), f2(0.0f), pairs_ok, second);
  }
  if (kOrdered) {
    reorder<NS>(dA, order);
    reorder<NS>(gam, order);
  }
  const int64_t to = (int64_t)span * g.B + b;
  store_states<NS>(g.part_A + (to * g.D + c) * g.N, g.N, n0, second, dA);
  if (span == 0 && g.grad_state_in)
    store_states<NS>(g.grad_state_in + ((int64_t)b * g.D + c) * g.N, g.N, n0, second, gam);
  if (pl == 0) {
    g.part_D[to * g.D + c] = sum_D.x;
    g.part_bias[to * g.D + c] = sum_bias.x;
    if (second) {
      g.part_D[to * g.D + c + 1] = sum_D.y;
      g.part_bias[to * g.D + c + 1] = sum_bias.y;
    }
  }
}

template <typename T, int NS, int P>
__global__ void __launch_bounds__(32 * kWarps, blocks_of(NS)) scan_bwd(const Args g, int64_t works) {
  extern __shared__ __align__(16) unsigned char scan_smem[];
  __shared__ uint32_t tmem_slot;
  const int warp = threadIdx.x >> 5;
  if (warp == 0) tmem_alloc(&tmem_slot, columns_of(NS));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  grid_dep_wait();
  const int64_t work = (int64_t)blockIdx.x * kWarps + warp;
  if (work < works)
    scan_back<T, NS, P>(g, work, scan_smem + warp * Smem<T, NS, P>::bytes, tmem + ((uint32_t)(warp * 32) << 16));
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, columns_of(NS));
}

// grad_B and grad_C: the warps' shares, in eight slices (every eighth, in order), then the
// slices in order; zero past a sequence's end.
template <typename T>
__global__ void __launch_bounds__(256) scan_sum_bc(const Args g, Mat gB, Mat gC, int blocks) {
  __shared__ float sum[2][8][32];
  grid_dep_wait();
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int64_t i = (int64_t)blockIdx.x * 32 + lane, all = (int64_t)g.B * g.T * g.G * g.N;
  const int64_t row = i / g.N;
  const int n = (int)(i - row * g.N);
  const int64_t token = row / g.G;
  const int grp = (int)(row - token * g.G), b = (int)(token / g.T), tok = (int)(token - (int64_t)b * g.T);
  const bool in = i < all;
  float vb = 0.0f, vc = 0.0f;
  if (in && tok < seq_len(g, b)) {
#pragma unroll 8
    for (int k = slice; k < blocks; k += 8) {
      vb += g.part_B[k * all + i];
      vc += g.part_C[k * all + i];
    }
  }
  sum[0][slice][lane] = vb;
  sum[1][slice][lane] = vc;
  __syncthreads();
  if (slice > 1 || !in) return;
  float v = sum[slice][0][lane];
#pragma unroll
  for (int k = 1; k < 8; ++k) v += sum[slice][k][lane];
  const Mat& m = slice ? gC : gB;
  Elem<T>::store1(static_cast<T*>(m.data) + b * m.sb + tok * m.st + grp * m.sg + n, v);
}

// grad_A, grad_D and grad_delta_bias: the spans' and sequences' shares in order.
__global__ void __launch_bounds__(256) scan_sum_par(const Args g, int rows, float* gA, float* gD, float* gbias) {
  grid_dep_wait();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, states = (int64_t)g.D * g.N;
  const float* p;
  float* out;
  int64_t width;
  if (i < states) p = g.part_A + i, out = gA + i, width = states;
  else if (i < states + g.D) p = g.part_D + (i - states), out = gD ? gD + (i - states) : nullptr, width = g.D;
  else if (i < states + 2 * g.D)
    p = g.part_bias + (i - states - g.D), out = gbias ? gbias + (i - states - g.D) : nullptr, width = g.D;
  else return;
  if (!out) return;
  float v = 0.0f;
#pragma unroll 4
  for (int k = 0; k < rows; ++k) v += p[k * width];
  *out = v;
}

struct BwdSpace {
  size_t ends, sums, bc, a, d, total;
};
BwdSpace bwd_space(const Args& g, const BwdPlan& p) {
  BwdSpace s;
  s.ends = p.cut.spans > 1 ? ends_bytes(g, p.cut.spans * p.cut.fine) : 0;
  s.sums = p.cut.spans > 1 ? sums_bytes(g, p.cut.spans * p.cut.fine) : 0;
  s.bc = round256((size_t)p.blocks * g.B * g.T * g.G * g.N * sizeof(float));
  s.a = round256((size_t)p.cut.spans * g.B * g.D * g.N * sizeof(float));
  s.d = round256((size_t)p.cut.spans * g.B * g.D * sizeof(float));
  s.total = s.ends + s.sums + 2 * s.bc + s.a + 2 * s.d;
  return s;
}

template <typename T, int NS, int P>
cudaError_t launch_main(const Args& g, int64_t works, cudaStream_t st) {
  const size_t smem = (size_t)kWarps * Smem<T, NS, P>::bytes;
  // with the kernel's static shared memory, past the limit that needs no asking
  const size_t ask = smem + 1024 > 48 * 1024 && smem <= 48 * 1024 ? 48 * 1024 + 16 : smem;
  const cudaError_t e = ensure_smem((const void*)scan_bwd<T, NS, P>, ask);
  if (e != cudaSuccess) return e;
  return launch_pdl(scan_bwd<T, NS, P>, dim3((unsigned)ceil_div(works, kWarps)), dim3(32 * kWarps), smem, st, g, works);
}

template <typename T>
cudaError_t launch_bwd(const Args& g, const BwdPlan& p, const Mat& gB, const Mat& gC, cudaStream_t st) {
  const int64_t works = warps_of(g, p.lay) * g.spans, all = (int64_t)g.B * g.T * g.G * g.N;
  if (works > 0x7fffffff || ceil_div(all, 32) > 0x7fffffff) return cudaErrorInvalidValue;
  const cudaError_t e = with_lay<false>(p.lay, [&](auto NS, auto P) {
    return launch_main<T, decltype(NS)::value, decltype(P)::value>(g, works, st);
  });
  if (e != cudaSuccess || all == 0) return e;
  return launch_pdl(scan_sum_bc<T>, dim3((unsigned)ceil_div(all, 32)), dim3(256), 0, st, g, gB, gC, p.blocks);
}

}  // namespace sscan
}  // namespace snn

using namespace snn::sscan;

extern "C" {

size_t snn_selective_scan_workspace_bytes(const snn_sscan_desc* desc, int backward) {
  if (!desc) return 0;
  snn_sscan_desc d = *desc;
  d.dtype = SNN_F32;
  d.softplus = 0;
  if (check_desc(&d) != SNN_OK) return 0;
  const Args g = base_args(&d);
  size_t n = fwd_bytes(g, fwd_plan(g));
  if (backward) {
    const size_t m = bwd_space(g, bwd_plan(g)).total;
    n = m > n ? m : n;
  }
  return n < 256 ? 256 : n;
}

snn_status_t snn_selective_scan_bwd(const snn_sscan_desc* desc, const snn_btc* u,
                                    const snn_btc* delta, const float* A, const snn_bthd* Bm,
                                    const snn_bthd* Cm, const float* D, const snn_btc* z,
                                    const float* delta_bias, const int32_t* seq_lens,
                                    const float* ckpt, const snn_btc* grad_y,
                                    const float* grad_state_out, const snn_btc* grad_u,
                                    const snn_btc* grad_delta, float* grad_A,
                                    const snn_bthd* grad_B, const snn_bthd* grad_C, float* grad_D,
                                    const snn_btc* grad_z, float* grad_delta_bias,
                                    float* grad_state_in, void* ws, size_t ws_bytes,
                                    snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  const bool any = desc->B > 0 && desc->T > 0;
  if (!A || !grad_A || (any && !ckpt)) return SNN_ERR_INVALID_ARG;
  if (grad_state_in && grad_state_in == grad_state_out) return SNN_ERR_INVALID_ARG;
  const void* ptrs[11] = {A, D, delta_bias, seq_lens, ckpt, grad_state_out, grad_A, grad_D, grad_delta_bias,
                          grad_state_in, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  Args g = base_args(desc);
  bool pair = g.Dg % 2 == 0;
  Mat gB, gC;
  const bool gate = z && z->data;
  if (any) {
    if (gate != (grad_z && grad_z->data)) return SNN_ERR_INVALID_ARG;
    if ((s = take(desc, u, &g.u, &pair)) != SNN_OK || (s = take(desc, delta, &g.delta, &pair)) != SNN_OK ||
        (gate && (s = take(desc, z, &g.z, &pair)) != SNN_OK) ||
        (s = take(desc, grad_y, &g.gy, &pair)) != SNN_OK || (s = take(desc, Bm, &g.Bm)) != SNN_OK ||
        (s = take(desc, Cm, &g.Cm)) != SNN_OK || (s = take(desc, grad_u, &g.gu, &pair)) != SNN_OK ||
        (s = take(desc, grad_delta, &g.gdelta, &pair)) != SNN_OK ||
        (gate && (s = take(desc, grad_z, &g.gz, &pair)) != SNN_OK) || (s = take(desc, grad_B, &gB)) != SNN_OK ||
        (s = take(desc, grad_C, &gC)) != SNN_OK)
      return s;
  }
  const BwdPlan plan = bwd_plan(g);
  const BwdSpace space = bwd_space(g, plan);
  if (!ws || ws_bytes < space.total) return SNN_ERR_WORKSPACE;
  g.pair_ok = pair;
  g.quads = quads(g, {&g.Bm, &g.Cm});
  put_cut(g, plan.cut);
  g.A = A;
  g.D_skip = D;
  g.bias = delta_bias;
  g.seq_lens = seq_lens;
  g.ckpt = const_cast<float*>(ckpt);
  g.grad_state_out = grad_state_out;
  g.grad_state_in = grad_state_in;
  unsigned char* w = static_cast<unsigned char*>(ws);
  g.ends = reinterpret_cast<float*>(w);
  w += space.ends;
  g.sums = reinterpret_cast<float2*>(w);
  w += space.sums;
  g.part_B = reinterpret_cast<float*>(w);
  w += space.bc;
  g.part_C = reinterpret_cast<float*>(w);
  w += space.bc;
  g.part_A = reinterpret_cast<float*>(w);
  w += space.a;
  g.part_D = reinterpret_cast<float*>(w);
  w += space.d;
  g.part_bias = reinterpret_cast<float*>(w);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (g.B > 0) {
    if (g.spans > 1) e = launch_back_ends(g, plan.lay, desc->dtype, st);
    if (e == cudaSuccess)
      e = desc->dtype == SNN_F32    ? launch_bwd<float>(g, plan, gB, gC, st)
          : desc->dtype == SNN_BF16 ? launch_bwd<__nv_bfloat16>(g, plan, gB, gC, st)
                                    : launch_bwd<__half>(g, plan, gB, gC, st);
  }
  if (e == cudaSuccess)
    e = snn::launch_pdl(scan_sum_par, dim3((unsigned)snn::ceil_div((int64_t)g.D * (g.N + 2), 256)), dim3(256), 0,
                        st, g, g.spans * g.B, grad_A, grad_D, grad_delta_bias);
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

}  // extern "C"
