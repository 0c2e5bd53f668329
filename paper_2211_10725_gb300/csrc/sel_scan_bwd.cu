// Selective scan, backward.  With dy = grad_y silu(z) (the gradient of the sum over states
// and of D u), and gamma the gradient that reaches h_t from later tokens:
//   gt = dy C_t + gamma;        gamma <- a_t gt
//   grad_C = sum over channels of dy h_t;      grad_B = sum over channels of gt x
//   w = sum_n gt B;  q = a_t gt h_{t-1};  r = sum_n q A
//   grad_u = s w + D dy;   grad_delta = (u w + r) softplus'(delta + bias)
//   grad_A = sum_t q s;    grad_D = sum_t dy u;   grad_z = grad_y (y before the gate) silu'(z)
// A block goes backwards through its span of the axis in tiles of the checkpoints'
// eight tokens, and in each tile in turns through its channel pairs: it takes the states
// of a turn from the checkpoint through the tile (they stay in registers), then gamma
// back through it.  A thread has the same states in every turn, so that grad_B and
// grad_C of the tile gather in its registers over the turns and meet over the
// threads once a tile; gamma and grad_A of every turn lie in shared memory.  The blocks' shares
// of grad_B, grad_C, grad_A, grad_D and grad_delta_bias are added by a second kernel in a
// fixed order.
#include "sel_scan.cuh"
#include "sel_scan_plan.cuh"

namespace snn {
namespace sscan {

constexpr int kAccStride = kThreads + 4;  // floats: rows of the threads' shares, apart by four banks

struct BwdPlan {
  Plan cut;
  int per_block, blocks;  // turns of a block; blocks of a group
};

BwdPlan bwd_plan(const Args& g) {
  BwdPlan p;
  const int turns = (int)ceil_div(g.pairs, kThreads / g.P);
  p.per_block = turns < 4 ? turns : 4;
  p.blocks = (int)ceil_div(turns, p.per_block);
  p.cut = cut(g.T, (int64_t)g.B * g.G * p.blocks, kSms * 3);
  return p;
}

// Shared memory: s and x, dy; B and C; the sums' parts (or the threads' shares of
// grad_B and grad_C); what stays over the tiles of a span.
size_t bwd_smem(const Args& g, int per_block) {
  const int cp = kThreads / g.P;
  const size_t parts = 3 * kCkpt * kThreads * sizeof(float2), acc = 32 * kAccStride * sizeof(float);
  return (size_t)kCkpt * cp * (sizeof(float4) + sizeof(float2)) + 2 * (size_t)kCkpt * g.P * 2 * sizeof(float4) +
         (parts > acc ? parts : acc) + (size_t)per_block * kThreads * (3 * 8 + 4) * sizeof(float);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) scan_bwd(const Args g) {
  extern __shared__ __align__(16) unsigned char scan_smem[];
  grid_dep_wait();
  const int P = g.P, cp = kThreads / P, R = kThreads / cp, N4 = kStates * P, M = g.per_block;
  float4* const sx = reinterpret_cast<float4*>(scan_smem);         // [8][cp]: s, x
  float4* const Bd = sx + kCkpt * cp;                              // [8][P][2]
  float4* const Cd = Bd + kCkpt * P * 2;
  float* const keep = reinterpret_cast<float*>(Cd + kCkpt * P * 2);  // [M][3][threads][8]: A, gamma, grad_A
  float4* const keep2 = reinterpret_cast<float4*>(keep + M * 3 * kThreads * 8);  // [M][threads]: grad_D, grad_delta_bias
  float2* const dys = reinterpret_cast<float2*>(keep2 + M * kThreads);  // [8][cp]
  float2* const yp = dys + kCkpt * cp;                             // [8][threads]
  float2* const wp = yp + kCkpt * kThreads;
  float2* const rp = wp + kCkpt * kThreads;
  float* const acc = reinterpret_cast<float*>(yp);                 // [32][kAccStride]

  const int turns = (g.pairs + cp - 1) / cp, nb = (turns + M - 1) / M;
  const int pb = blockIdx.x % nb, rest = blockIdx.x / nb, grp = rest % g.G, b = rest / g.G;
  const int span = blockIdx.y, len = seq_len(g, b), first = span * g.span;
  const int last = first + g.span < g.T ? first + g.span : g.T;
  const int stop = last < len ? last : len;
  const int tiles = stop > first ? (stop - first + kCkpt - 1) / kCkpt : 0;
  const int t = threadIdx.x, pl = t % P, pc = t / P;
  const int pr = t % cp, row = t / cp;
  const bool pairs_ok = g.pair_ok;
  const int64_t own_all = (int64_t)g.B * g.G * g.pairs * P;
  auto keep_at = [&](int m, int k) { return keep + ((m * 3 + k) * kThreads + t) * 8; };

  for (int m = 0; m < M; ++m) {
    const int pair = (pb * M + m) * cp + pc;
    float2 A2[kStates], gam[kStates];
#pragma unroll
    for (int q = 0; q < kStates; ++q) A2[q] = gam[q] = f2(0.0f);
    if (pc < cp && pair < g.pairs) {
      const int c = grp * g.Dg + 2 * pair;
      const bool second = 2 * pair + 1 < g.Dg;
      const int64_t own = (((int64_t)b * g.G + grp) * g.pairs + pair) * P + pl;
      load_states(g.A + (int64_t)c * g.N, g.N, pl * kStates, second, A2);
#pragma unroll
      for (int q = 0; q < kStates; ++q) A2[q] = mul2(A2[q], f2(kLog2E));
      if (g.grad_state_out)
        load_states(g.grad_state_out + ((int64_t)b * g.D + c) * g.N, g.N, pl * kStates, second, gam);
      for (int i = g.spans - 1; i > span; --i) {
        float2 e[kStates];
        load_own(g.ends + ((int64_t)i * own_all + own) * 2 * kStates, e);
        const float2 s = g.sums[((int64_t)i * g.B * g.G + rest) * g.pairs + pair];
#pragma unroll
        for (int q = 0; q < kStates; ++q) gam[q] = fma2(ex2(mul2(s, A2[q])), gam[q], e[q]);
      }
    }
    store_own(keep_at(m, 0), A2);
    store_own(keep_at(m, 1), gam);
#pragma unroll
    for (int q = 0; q < kStates; ++q) gam[q] = f2(0.0f);
    store_own(keep_at(m, 2), gam);
    keep2[m * kThreads + t] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  }

  const int n_bc = t % N4, row_bc = t / N4, R_bc = kThreads / N4;
  for (int tile = tiles - 1; tile >= 0; --tile) {
    const int t0 = first + tile * kCkpt;
    if (row_bc < R_bc) {
      for (int tok = row_bc; tok < kCkpt; tok += R_bc) {
        float vb = 0.0f, vc = 0.0f;
        const int now = t0 + tok;
        if (n_bc < g.N && now < stop) {
          vb = Elem<T>::load1(static_cast<const T*>(g.Bm.data) + b * g.Bm.sb + now * g.Bm.st + grp * g.Bm.sg + n_bc);
          vc = Elem<T>::load1(static_cast<const T*>(g.Cm.data) + b * g.Cm.sb + now * g.Cm.st + grp * g.Cm.sg + n_bc);
        }
        reinterpret_cast<float2*>(Bd)[tok * N4 + n_bc] = f2(vb);
        reinterpret_cast<float2*>(Cd)[tok * N4 + n_bc] = f2(vc);
      }
    }
    float accB[kCkpt][kStates], accC[kCkpt][kStates];
#pragma unroll
    for (int i = 0; i < kCkpt; ++i)
#pragma unroll
      for (int q = 0; q < kStates; ++q) accB[i][q] = accC[i][q] = 0.0f;

    for (int m = 0; m < M; ++m) {
      const int pair0 = (pb * M + m) * cp;
      if (pair0 >= g.pairs) break;
      const bool loads = row < R && pair0 + pr < g.pairs;
      const int c = grp * g.Dg + 2 * (pair0 + pr);
      const bool second = 2 * (pair0 + pr) + 1 < g.Dg;
      auto at = [&](const Seq& x, int tok) { return static_cast<T*>(x.data) + b * x.sb + tok * x.st + c; };
      auto value = [&](const Seq& x, int tok) {
        Raw<T> r;
        r.load(at(x, tok), pairs_ok, second);
        return r.get();
      };
      float2 bias = f2(0.0f), skip = f2(0.0f);
      if (loads) {
        if (g.bias) bias = make_float2(g.bias[c], second ? g.bias[c + 1] : 0.0f);
        if (g.D_skip) skip = make_float2(g.D_skip[c], second ? g.D_skip[c + 1] : 0.0f);
        for (int tok = row; tok < kCkpt; tok += R) {
          float2 s = f2(0.0f), x = f2(0.0f), dy = f2(0.0f);
          const int now = t0 + tok;
          if (now < stop) {
            s = step_of(value(g.delta, now), bias, g.softplus);
            x = mul2(s, value(g.u, now));
            dy = value(g.gy, now);
            if (g.z.data) {
              const float2 z = value(g.z, now);
              dy = mul2(dy, mul2(z, sigmoid<T>(z)));
            }
            if (!second) s.y = x.y = dy.y = 0.0f;
          }
          sx[tok * cp + pr] = make_float4(s.x, s.y, x.x, x.y);
          dys[tok * cp + pr] = dy;
        }
      }
      __syncthreads();
      const int pair = pair0 + pc;
      if (pc < cp && pair < g.pairs) {
        float2 A2[kStates], h[kCkpt + 1][kStates], gam[kStates], dA[kStates];
        const int64_t at_tile = (int64_t)b * ((g.T + kCkpt - 1) / kCkpt) + t0 / kCkpt;
        load_own(g.ckpt + (((at_tile * g.G + grp) * g.pairs + pair) * P + pl) * 2 * kStates, h[0]);
        load_own(keep_at(m, 0), A2);
#pragma unroll
        for (int i = 0; i < kCkpt; ++i) {
          const float4 v = sx[i * cp + pc];
          const float2 s = make_float2(v.x, v.y), x = make_float2(v.z, v.w), dy = dys[i * cp + pc];
          const float2* bp = reinterpret_cast<const float2*>(Bd) + (i * P + pl) * 4;
          const float2* cq = reinterpret_cast<const float2*>(Cd) + (i * P + pl) * 4;
          float2 y = f2(0.0f);
#pragma unroll
          for (int q = 0; q < kStates; ++q) {
            h[i + 1][q] = fma2(ex2(mul2(s, A2[q])), h[i][q], mul2(x, bp[q]));
            y = fma2(cq[q], h[i + 1][q], y);
            accC[i][q] = fmaf(dy.x, h[i + 1][q].x, accC[i][q]);
            accC[i][q] = fmaf(dy.y, h[i + 1][q].y, accC[i][q]);
          }
          yp[i * kThreads + t] = y;
        }
        load_own(keep_at(m, 1), gam);
        load_own(keep_at(m, 2), dA);
#pragma unroll
        for (int i = kCkpt - 1; i >= 0; --i) {
          const float4 v = sx[i * cp + pc];
          const float2 s = make_float2(v.x, v.y), x = make_float2(v.z, v.w), dy = dys[i * cp + pc];
          const float2* bp = reinterpret_cast<const float2*>(Bd) + (i * P + pl) * 4;
          const float2* cq = reinterpret_cast<const float2*>(Cd) + (i * P + pl) * 4;
          float2 w = f2(0.0f), r = f2(0.0f);
#pragma unroll
          for (int q = 0; q < kStates; ++q) {
            const float2 gt = fma2(dy, cq[q], gam[q]);
            accB[i][q] = fmaf(gt.x, x.x, accB[i][q]);
            accB[i][q] = fmaf(gt.y, x.y, accB[i][q]);
            w = fma2(gt, bp[q], w);
            gam[q] = mul2(ex2(mul2(s, A2[q])), gt);
            const float2 qq = mul2(gam[q], h[i][q]);
            r = fma2(qq, A2[q], r);
            dA[q] = fma2(qq, s, dA[q]);
          }
          wp[i * kThreads + t] = w;
          rp[i * kThreads + t] = r;
        }
        store_own(keep_at(m, 1), gam);
        store_own(keep_at(m, 2), dA);
      }
      __syncthreads();
      if (loads) {
        float4 sums = keep2[m * kThreads + t];
        for (int tok = row; tok < kCkpt; tok += R) {
          const int now = t0 + tok;
          if (now >= last) break;
          float2 gu = f2(0.0f), gd = f2(0.0f), gz = f2(0.0f);
          if (now < stop) {
            const int i = tok * kThreads + pr * P;
            float2 y = yp[i], w = wp[i], r = rp[i];
            for (int k = 1; k < P; ++k) y = add2(y, yp[i + k]), w = add2(w, wp[i + k]), r = add2(r, rp[i + k]);
            const float4 v = sx[tok * cp + pr];
            const float2 s = make_float2(v.x, v.y), dy = dys[tok * cp + pr], u = value(g.u, now);
            gu = fma2(s, w, mul2(skip, dy));
            gd = fma2(u, w, mul2(r, f2(0.69314718055994530942f)));  // r holds A log2(e)
            if (g.softplus) gd = mul2(gd, sigmoid<T>(add2(value(g.delta, now), bias)));
            if (g.z.data) {
              const float2 z = value(g.z, now), sig = sigmoid<T>(z);
              const float2 slope = fma2(mul2(z, sig), fma2(sig, f2(-1.0f), f2(1.0f)), sig);
              gz = mul2(mul2(value(g.gy, now), fma2(skip, u, y)), slope);
            }
            sums.x = fmaf(dy.x, u.x, sums.x);
            sums.y = fmaf(dy.y, u.y, sums.y);
            sums.z += gd.x;
            sums.w += gd.y;
          }
          put_pair(at(g.gu, now), gu, pairs_ok, second);
          put_pair(at(g.gdelta, now), gd, pairs_ok, second);
          if (g.z.data) put_pair(at(g.gz, now), gz, pairs_ok, second);
        }
        keep2[m * kThreads + t] = sums;
      }
    }
    // grad_B and grad_C of the tile: the threads' shares, pair after pair
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kCkpt; ++i)
#pragma unroll
        for (int q = 0; q < kStates; ++q)
          acc[(i * kStates + q) * kAccStride + t] = pc < cp ? (which ? accC[i][q] : accB[i][q]) : 0.0f;
      __syncthreads();
      float* part = which ? g.part_C : g.part_B;
      for (int o = t; o < kCkpt * N4; o += kThreads) {
        const int i = o / N4, n = o - i * N4;
        const float* p = acc + (i * kStates + (n & 3)) * kAccStride + (n >> 2);
        float v = p[0];
        for (int k = 1; k < cp; ++k) v += p[k * P];
        if (n < g.N && t0 + i < stop)
          part[((((int64_t)pb * g.B + b) * g.T + t0 + i) * g.G + grp) * g.N + n] = v;
      }
    }
    __syncthreads();
  }

  for (int m = 0; m < M; ++m) {
    const int pair0 = (pb * M + m) * cp, pair = pair0 + pc;
    const int64_t to = (int64_t)span * g.B + b;
    if (pc < cp && pair < g.pairs) {
      const int c = grp * g.Dg + 2 * pair;
      const bool second = 2 * pair + 1 < g.Dg;
      float2 v[kStates];
      load_own(keep_at(m, 2), v);
      store_states(g.part_A + (to * g.D + c) * g.N, g.N, pl * kStates, second, v);
      if (span == 0 && g.grad_state_in) {
        load_own(keep_at(m, 1), v);
        store_states(g.grad_state_in + ((int64_t)b * g.D + c) * g.N, g.N, pl * kStates, second, v);
      }
    }
    // places past the sequence's end
    if (row < R && pair0 + pr < g.pairs) {
      const int c = grp * g.Dg + 2 * (pair0 + pr);
      const bool second = 2 * (pair0 + pr) + 1 < g.Dg;
      for (int now = first + tiles * kCkpt + row; now < last; now += R) {
        const int64_t chan = c;
        put_pair(static_cast<T*>(g.gu.data) + b * g.gu.sb + now * g.gu.st + chan, f2(0.0f), pairs_ok, second);
        put_pair(static_cast<T*>(g.gdelta.data) + b * g.gdelta.sb + now * g.gdelta.st + chan, f2(0.0f), pairs_ok, second);
        if (g.z.data)
          put_pair(static_cast<T*>(g.gz.data) + b * g.gz.sb + now * g.gz.st + chan, f2(0.0f), pairs_ok, second);
      }
    }
    // grad_D and grad_delta_bias: the rows of a pair, in order
    __syncthreads();
    if (row == 0 && pr < cp && pair0 + pr < g.pairs) {
      const int c = grp * g.Dg + 2 * (pair0 + pr);
      const bool second = 2 * (pair0 + pr) + 1 < g.Dg;
      float4 v = keep2[m * kThreads + pr];
      for (int k = 1; k < R; ++k) {
        const float4 w = keep2[m * kThreads + k * cp + pr];
        v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
      }
      g.part_D[to * g.D + c] = v.x;
      g.part_bias[to * g.D + c] = v.z;
      if (second) {
        g.part_D[to * g.D + c + 1] = v.y;
        g.part_bias[to * g.D + c + 1] = v.w;
      }
    }
  }
}

// grad_B and grad_C: the blocks' shares in order; zero past a sequence's end.
template <typename T>
__global__ void __launch_bounds__(256) scan_sum_bc(const Args g, Mat gB, Mat gC, int blocks) {
  grid_dep_wait();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = (int64_t)g.B * g.T * g.G * g.N;
  if (i >= all) return;
  const int n = (int)(i % g.N);
  int64_t rest = i / g.N;
  const int grp = (int)(rest % g.G);
  rest /= g.G;
  const int tok = (int)(rest % g.T), b = (int)(rest / g.T);
  float vb = 0.0f, vc = 0.0f;
  if (tok < seq_len(g, b)) {
    for (int k = 0; k < blocks; ++k) {
      vb += g.part_B[k * all + i];
      vc += g.part_C[k * all + i];
    }
  }
  Elem<T>::store1(static_cast<T*>(gB.data) + b * gB.sb + tok * gB.st + grp * gB.sg + n, vb);
  Elem<T>::store1(static_cast<T*>(gC.data) + b * gC.sb + tok * gC.st + grp * gC.sg + n, vc);
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
  s.ends = p.cut.spans > 1 ? ends_bytes(g, p.cut.spans) : 0;
  s.sums = p.cut.spans > 1 ? sums_bytes(g, p.cut.spans) : 0;
  s.bc = round256((size_t)p.blocks * g.B * g.T * g.G * g.N * sizeof(float));
  s.a = round256((size_t)p.cut.spans * g.B * g.D * g.N * sizeof(float));
  s.d = round256((size_t)p.cut.spans * g.B * g.D * sizeof(float));
  s.total = s.ends + s.sums + 2 * s.bc + s.a + 2 * s.d;
  return s;
}

template <typename T>
cudaError_t launch_bwd(const Args& g, const BwdPlan& p, const Mat& gB, const Mat& gC, cudaStream_t st) {
  const size_t smem = bwd_smem(g, p.per_block);
  cudaError_t e = ensure_smem((const void*)scan_bwd<T>, smem);
  if (e != cudaSuccess) return e;
  const int64_t blocks = (int64_t)g.B * g.G * p.blocks, all = (int64_t)g.B * g.T * g.G * g.N;
  if (blocks > 0x7fffffff || ceil_div(all, 256) > 0x7fffffff) return cudaErrorInvalidValue;
  e = launch_pdl(scan_bwd<T>, dim3((unsigned)blocks, (unsigned)g.spans), dim3(kThreads), smem, st, g);
  if (e != cudaSuccess || all == 0) return e;
  return launch_pdl(scan_sum_bc<T>, dim3((unsigned)ceil_div(all, 256)), dim3(256), 0, st, g, gB, gC, p.blocks);
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
  g.spans = plan.cut.spans;
  g.span = plan.cut.span;
  g.per_block = plan.per_block;
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
    if (g.spans > 1) e = launch_back_ends(g, desc->dtype, st);
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
