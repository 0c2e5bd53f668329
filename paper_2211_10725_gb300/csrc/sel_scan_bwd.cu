// Selective scan, backward.  With dy = grad_y silu(z) (the gradient of the sum over states
// and of D u), and gamma the gradient that reaches h_t from later tokens:
//   gt = dy C_t + gamma;        gamma <- a_t gt
//   grad_C = sum over channels of dy h_t;      grad_B = sum over channels of gt x
//   w = sum_n gt B;  q = a_t gt h_{t-1};  r = sum_n q A
//   grad_u = s w + D dy;   grad_delta = (u w + r) softplus'(delta + bias)
//   grad_A = sum_t q s;    grad_D = sum_t dy u;   grad_z = grad_y (y before the gate) silu'(z)
// A warp goes backwards through its span of the axis in tiles of the checkpoints'
// eight tokens, and in each tile in turns through its channel pairs: it takes the states
// of a turn from the checkpoint through the tile (they stay in registers), then gamma
// back through it.  A thread has the same states in every turn, so that grad_B and
// grad_C of the tile gather in its registers over the turns and meet over the
// threads once a tile; gamma and grad_A of every turn lie in shared memory.  The warps' shares
// of grad_B, grad_C, grad_A, grad_D and grad_delta_bias are added by a second kernel in a
// fixed order.
#include "sel_scan.cuh"
#include "sel_scan_plan.cuh"

namespace snn {
namespace sscan {

constexpr int kTurns = 4;        // of a warp in a tile, at most
constexpr int kAccStride = 36;   // floats between the rows of the threads' shares: 32 and four banks

struct BwdPlan {
  Plan cut;
  int per_block, blocks;  // turns of a warp; warps of a group
};

BwdPlan bwd_plan(const Args& g) {
  BwdPlan p;
  const int turns = (int)ceil_div(g.pairs, 32 / g.P);
  p.per_block = turns < kTurns ? turns : kTurns;
  p.blocks = (int)ceil_div(turns, p.per_block);
  p.cut = cut(g.T, (int64_t)g.B * g.G * p.blocks, kSms * 8, 3);
  return p;
}

// Shared memory of a warp: s and x; slopes; dy; B and C; the sums' parts (or the threads'
// shares of grad_B and grad_C); what stays over the tiles of a span.
__host__ __device__ constexpr int bwd_smem(int P, int turns) {
  return kTile * (32 / P) * (2 * (int)sizeof(float4) + (int)sizeof(float2)) +
         2 * kTile * P * kStates * (int)sizeof(float2) + 3 * kTile * 32 * (int)sizeof(float2) +
         turns * 32 * (3 * 8 + 4) * (int)sizeof(float);
}

template <typename T, int PT>
__global__ void __launch_bounds__(32) scan_bwd(const Args g) {
  extern __shared__ __align__(16) unsigned char scan_smem[];
  constexpr int kUnits = units_of(PT);
  grid_dep_wait();
  const int P = PT ? PT : g.P, PW = 32 / P, R = 32 / PW, N4 = kStates * P, M = g.per_block, lane = threadIdx.x;
  float4* const sx = reinterpret_cast<float4*>(scan_smem);         // [kTile][PW]: s, x
  float4* const slopes = sx + kTile * PW;                          // [kTile][PW]: softplus', grad_y silu'
  float2* const Bd = reinterpret_cast<float2*>(slopes + kTile * PW);  // [kTile][P][4]
  float2* const Cd = Bd + kTile * N4;
  float* const keep = reinterpret_cast<float*>(Cd + kTile * N4);   // [M][3][32][8]: A, gamma, grad_A
  float4* const keep2 = reinterpret_cast<float4*>(keep + M * 3 * 32 * 8);  // [M][32]: grad_D, grad_delta_bias
  float2* const yp = reinterpret_cast<float2*>(keep2 + M * 32);    // [kTile][32]
  float2* const wp = yp + kTile * 32;
  float2* const rp = wp + kTile * 32;
  float2* const dys = rp + kTile * 32;                             // [kTile][PW]
  float* const acc = reinterpret_cast<float*>(yp);                 // [32][kAccStride]

  const int turns = (g.pairs + PW - 1) / PW, nb = (turns + M - 1) / M;
  const int pb = blockIdx.x % nb, rest = blockIdx.x / nb, grp = rest % g.G, b = rest / g.G;
  const int span = blockIdx.y, len = seq_len(g, b), first = span * g.span;
  const int last = first + g.span < g.T ? first + g.span : g.T;
  const int stop = last < len ? last : len;
  const int tiles = stop > first ? (stop - first + kTile - 1) / kTile : 0;
  const int pl = lane % P, pc = lane / P, pr = lane % PW, row = lane / PW;
  const bool pairs_ok = g.pair_ok, gate = g.z.data != nullptr;
  const int64_t own_all = (int64_t)g.B * g.G * g.pairs * P;
  auto keep_at = [&](int m, int k) { return keep + ((m * 3 + k) * 32 + lane) * 8; };

  for (int m = 0; m < M; ++m) {
    const int pair = (pb * M + m) * PW + pc;
    float2 A2[kStates], gam[kStates];
#pragma unroll
    for (int q = 0; q < kStates; ++q) A2[q] = gam[q] = f2(0.0f);
    if (pc < PW && pair < g.pairs) {
      const int c = grp * g.Dg + 2 * pair;
      const bool second = 2 * pair + 1 < g.Dg;
      const int64_t own = (((int64_t)b * g.G + grp) * g.pairs + pair) * P + pl;
      load_states(g.A + (int64_t)c * g.N, g.N, pl * kStates, second, A2);
#pragma unroll
      for (int q = 0; q < kStates; ++q) A2[q] = mul2(A2[q], f2(kLog2E));
      if (g.grad_state_out)
        load_states(g.grad_state_out + ((int64_t)b * g.D + c) * g.N, g.N, pl * kStates, second, gam);
#pragma unroll 2
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
    keep2[m * 32 + lane] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  }

  const int c0 = grp * g.Dg + 2 * (pb * M * PW + pr);   // the first turn's channel where tokens are loaded and stored
  auto base = [&](const Seq& x) { return static_cast<T*>(x.data) + b * x.sb + c0; };
  const T *const pu = base(g.u), *const pd = base(g.delta), *const pg = base(g.gy), *const pz = base(g.z);
  T *const ou = base(g.gu), *const od = base(g.gdelta), *const oz = base(g.gz);
  const int64_t ckpt_step = (int64_t)g.G * g.pairs * P * 2 * kStates;

  for (int tile = tiles - 1; tile >= 0; --tile) {
    const int t0 = first + tile * kTile;
    load_tile<T>(g, g.Bm, Bd, P, b, grp, t0, stop, lane);
    load_tile<T>(g, g.Cm, Cd, P, b, grp, t0, stop, lane);
    const float* const ckpt = g.ckpt + ((int64_t)b * ((g.T + kTile - 1) / kTile) + t0 / kTile) * ckpt_step +
                              (((int64_t)grp * g.pairs + pb * M * PW + pc) * P + pl) * 2 * kStates;
    float accB[kTile][kStates], accC[kTile][kStates];
#pragma unroll
    for (int i = 0; i < kTile; ++i)
#pragma unroll
      for (int q = 0; q < kStates; ++q) accB[i][q] = accC[i][q] = 0.0f;

#pragma unroll 1
    for (int m = 0; m < M; ++m) {
      const int pair0 = (pb * M + m) * PW, off = 2 * m * PW;
      if (pair0 >= g.pairs) break;
      const bool loads = row < R && pair0 + pr < g.pairs, scans = pc < PW && pair0 + pc < g.pairs;
      const bool second = 2 * (pair0 + pr) + 1 < g.Dg;
      float2 h[kTile + 1][kStates];
      if (scans) load_own(ckpt + (int64_t)m * PW * P * 2 * kStates, h[0]);
      Raw<T> raw_u[kUnits];
      float2 bias = f2(0.0f), skip = f2(0.0f);
      if (loads) {
        const int c = c0 + off;
        if (g.bias) bias = make_float2(g.bias[c], second ? g.bias[c + 1] : 0.0f);
        if (g.D_skip) skip = make_float2(g.D_skip[c], second ? g.D_skip[c + 1] : 0.0f);
        Raw<T> raw_d[kUnits], raw_g[kUnits], raw_z[kUnits];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
          const int tok = row + k * R, now = t0 + tok;
          raw_u[k].clear();
          raw_d[k].clear();
          raw_g[k].clear();
          raw_z[k].clear();
          if (tok < kTile && now < stop) {
            raw_u[k].load(pu + now * g.u.st + off, pairs_ok, second);
            raw_d[k].load(pd + now * g.delta.st + off, pairs_ok, second);
            raw_g[k].load(pg + now * g.gy.st + off, pairs_ok, second);
            if (gate) raw_z[k].load(pz + now * g.z.st + off, pairs_ok, second);
          }
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
          const int tok = row + k * R;
          if (tok < kTile) {
            float2 s = f2(0.0f), x = f2(0.0f), dy = f2(0.0f), slope = f2(0.0f), gz = f2(0.0f);
            if (t0 + tok < stop) {
              s = step_of(add2(raw_d[k].get(), bias), g.softplus, &slope);
              x = mul2(s, raw_u[k].get());
              dy = raw_g[k].get();
              if (gate) {
                const float2 z = raw_z[k].get(), sig = sigmoid<T>(z), zs = mul2(z, sig);
                gz = mul2(dy, fma2(zs, fma2(sig, f2(-1.0f), f2(1.0f)), sig));
                dy = mul2(dy, zs);
              }
              if (!second) s.y = x.y = dy.y = 0.0f;
            }
            sx[tok * PW + pr] = make_float4(s.x, s.y, x.x, x.y);
            slopes[tok * PW + pr] = make_float4(slope.x, slope.y, gz.x, gz.y);
            dys[tok * PW + pr] = dy;
          }
        }
      }
      __syncwarp();
      if (scans) {
        float2 A2[kStates], gam[kStates], dA[kStates];
        load_own(keep_at(m, 0), A2);
#pragma unroll
        for (int i = 0; i < kTile; ++i) {
          const float4 v = sx[i * PW + pc];
          const float2 s = make_float2(v.x, v.y), x = make_float2(v.z, v.w), dy = dys[i * PW + pc];
          float2 bc[kStates];
          load_own(reinterpret_cast<const float*>(Bd + (i * P + pl) * kStates), bc);
#pragma unroll
          for (int q = 0; q < kStates; ++q) {
            h[i + 1][q] = fma2(ex2(mul2(s, A2[q])), h[i][q], mul2(x, bc[q]));
            accC[i][q] = fmaf(dy.x, h[i + 1][q].x, accC[i][q]);
            accC[i][q] = fmaf(dy.y, h[i + 1][q].y, accC[i][q]);
          }
          load_own(reinterpret_cast<const float*>(Cd + (i * P + pl) * kStates), bc);
          float2 y = mul2(bc[0], h[i + 1][0]);
#pragma unroll
          for (int q = 1; q < kStates; ++q) y = fma2(bc[q], h[i + 1][q], y);
          yp[i * 32 + lane] = y;
        }
        load_own(keep_at(m, 1), gam);
        load_own(keep_at(m, 2), dA);
#pragma unroll
        for (int i = kTile - 1; i >= 0; --i) {
          const float4 v = sx[i * PW + pc];
          const float2 s = make_float2(v.x, v.y), x = make_float2(v.z, v.w), dy = dys[i * PW + pc];
          float2 bc[kStates], w, r;
          load_own(reinterpret_cast<const float*>(Cd + (i * P + pl) * kStates), bc);
#pragma unroll
          for (int q = 0; q < kStates; ++q) gam[q] = fma2(dy, bc[q], gam[q]);
          load_own(reinterpret_cast<const float*>(Bd + (i * P + pl) * kStates), bc);
#pragma unroll
          for (int q = 0; q < kStates; ++q) {
            accB[i][q] = fmaf(gam[q].x, x.x, accB[i][q]);
            accB[i][q] = fmaf(gam[q].y, x.y, accB[i][q]);
            w = q ? fma2(gam[q], bc[q], w) : mul2(gam[q], bc[q]);
            gam[q] = mul2(ex2(mul2(s, A2[q])), gam[q]);
            const float2 qq = mul2(gam[q], h[i][q]);
            r = q ? fma2(qq, A2[q], r) : mul2(qq, A2[q]);
            dA[q] = fma2(qq, s, dA[q]);
          }
          wp[i * 32 + lane] = w;
          rp[i * 32 + lane] = r;
        }
        store_own(keep_at(m, 1), gam);
        store_own(keep_at(m, 2), dA);
      }
      __syncwarp();
      if (loads) {
        float4 sums = keep2[m * 32 + lane];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
          const int tok = row + k * R, now = t0 + tok;
          if (tok < kTile && now < last) {
            float2 gu = f2(0.0f), gd = f2(0.0f), gz = f2(0.0f);
            if (now < stop) {
              const int i = tok * 32 + pr * P;
              const float2 w = sum_parts<PT>(wp + i, P), r = sum_parts<PT>(rp + i, P);
              const float4 v = sx[tok * PW + pr], sl = slopes[tok * PW + pr];
              const float2 s = make_float2(v.x, v.y), dy = dys[tok * PW + pr], u = raw_u[k].get();
              gu = fma2(s, w, mul2(skip, dy));
              gd = fma2(u, w, mul2(r, f2(0.69314718055994530942f)));  // r holds A log2(e)
              gd = mul2(gd, make_float2(sl.x, sl.y));
              if (gate) gz = mul2(make_float2(sl.z, sl.w), fma2(skip, u, sum_parts<PT>(yp + i, P)));
              const float2 d = fma2(dy, u, make_float2(sums.x, sums.y)), e = add2(gd, make_float2(sums.z, sums.w));
              sums = make_float4(d.x, d.y, e.x, e.y);
            }
            put_pair(ou + now * g.gu.st + off, gu, pairs_ok, second);
            put_pair(od + now * g.gdelta.st + off, gd, pairs_ok, second);
            if (gate) put_pair(oz + now * g.gz.st + off, gz, pairs_ok, second);
          }
        }
        keep2[m * 32 + lane] = sums;
      }
    }
    // grad_B and grad_C of the tile: the threads' shares, pair after pair
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kTile; ++i)
#pragma unroll
        for (int q = 0; q < kStates; ++q) acc[(i * kStates + q) * kAccStride + lane] = which ? accC[i][q] : accB[i][q];
      __syncwarp();
      float* part = (which ? g.part_C : g.part_B) + ((((int64_t)pb * g.B + b) * g.T + t0) * g.G + grp) * g.N;
      for (int o = lane; o < kTile * N4; o += 32) {
        const int i = o / N4, n = o - i * N4;
        const float* p = acc + (i * kStates + (n & 3)) * kAccStride + (n >> 2);
        float v = p[0];
        for (int k = 1; k < PW; ++k) v += p[k * P];
        if (n < g.N && t0 + i < stop) part[(int64_t)i * g.G * g.N + n] = v;
      }
    }
    __syncwarp();
  }

  for (int m = 0; m < M; ++m) {
    const int pair0 = (pb * M + m) * PW, pair = pair0 + pc, off = 2 * m * PW;
    const int64_t to = (int64_t)span * g.B + b;
    if (pc < PW && pair < g.pairs) {
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
    __syncwarp();
    if (row < R && pair0 + pr < g.pairs) {
      const int c = c0 + off;
      const bool second = 2 * (pair0 + pr) + 1 < g.Dg;
      // places past the sequence's end
      for (int now = first + tiles * kTile + row; now < last; now += R) {
        put_pair(ou + now * g.gu.st + off, f2(0.0f), pairs_ok, second);
        put_pair(od + now * g.gdelta.st + off, f2(0.0f), pairs_ok, second);
        if (gate) put_pair(oz + now * g.gz.st + off, f2(0.0f), pairs_ok, second);
      }
      // grad_D and grad_delta_bias: the rows of a pair, in order
      if (row == 0) {
        float4 v = keep2[m * 32 + pr];
        for (int k = 1; k < R; ++k) {
          const float4 w = keep2[m * 32 + k * PW + pr];
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
}

// grad_B and grad_C: the warps' shares in order; zero past a sequence's end.
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

template <typename T, int PT>
cudaError_t launch_main(const Args& g, const BwdPlan& p, int64_t blocks, cudaStream_t st) {
  const size_t smem = bwd_smem(g.P, p.per_block);
  const cudaError_t e = ensure_smem((const void*)scan_bwd<T, PT>, smem);
  if (e != cudaSuccess) return e;
  return launch_pdl(scan_bwd<T, PT>, dim3((unsigned)blocks, (unsigned)g.spans), dim3(32), smem, st, g);
}

template <typename T>
cudaError_t launch_bwd(const Args& g, const BwdPlan& p, const Mat& gB, const Mat& gC, cudaStream_t st) {
  const int64_t blocks = (int64_t)g.B * g.G * p.blocks, all = (int64_t)g.B * g.T * g.G * g.N;
  if (blocks > 0x7fffffff || ceil_div(all, 256) > 0x7fffffff) return cudaErrorInvalidValue;
  const cudaError_t e = g.P == 4 ? launch_main<T, 4>(g, p, blocks, st) : launch_main<T, 0>(g, p, blocks, st);
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
  g.quads = quads(g, {&g.Bm, &g.Cm});
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
