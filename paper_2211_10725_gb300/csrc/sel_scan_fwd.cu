// Selective scan over whole sequences, and the spans' ends for it and for its
// backward.  A warp goes through its span of the axis in tiles of eight tokens:
//   1. its threads turn delta and u of the tile into s and x = s u (shared memory)
//      and spread B and C, each value twice, so that it meets both channels of a pair;
//   2. every thread takes its four states of a pair through the tile's tokens and
//      leaves its part of the sum over states;
//   3. the parts are added, skipped over by D u, gated and stored.
// The next tile's inputs are loaded into registers before 2.
#include "sel_scan.cuh"
#include "sel_scan_plan.cuh"

namespace snn {
namespace sscan {

enum Mode {
  kFull = 0,   // outputs
  kEnds = 1,   // what a span adds to the state after it
  kBack = 2    // what a span adds to the gradient of the state before it
};

// Shared memory of a warp.
__host__ __device__ constexpr int fwd_smem(int P, int mode) {
  return kTile * (32 / P) * (int)sizeof(float4) + (mode == kFull ? 2 : 1) * kTile * P * kStates * (int)sizeof(float2) +
         (mode == kFull ? kTile * 32 * (int)sizeof(float2) : 0);
}

// PT: threads of a pair, 0 where only the call knows them
template <typename T, int MODE, int PT>
__global__ void __launch_bounds__(32) scan_fwd(const Args g) {
  extern __shared__ __align__(16) unsigned char scan_smem[];
  constexpr int kUnits = units_of(PT);   // channel pairs of tokens that a thread loads for a tile
  grid_dep_wait();
  const int P = PT ? PT : g.P, PW = 32 / P, R = 32 / PW, lane = threadIdx.x;
  float4* const sx = reinterpret_cast<float4*>(scan_smem);               // [kTile][PW]: s, x
  float2* const Bd = reinterpret_cast<float2*>(sx + kTile * PW);         // [kTile][P][4]; C where B is not used
  float2* const Cd = MODE == kFull ? Bd + kTile * P * kStates : Bd;
  float2* const yp = Cd + kTile * P * kStates;                           // [kTile][32]

  const int nb = (g.pairs + PW - 1) / PW;
  const int pb = blockIdx.x % nb, rest = blockIdx.x / nb, grp = rest % g.G, b = rest / g.G;
  const int span = blockIdx.y + (MODE == kBack ? 1 : 0);
  const int len = seq_len(g, b), first = span * g.span;
  const int last = first + g.span < g.T ? first + g.span : g.T;
  const int pair0 = pb * PW;

  // the thread's states
  const int pl = lane % P, pc = lane / P, pair = pair0 + pc;
  const bool scans = pc < PW && pair < g.pairs;
  const int64_t own = (((int64_t)b * g.G + grp) * g.pairs + pair) * P + pl;
  const int64_t own_all = (int64_t)g.B * g.G * g.pairs * P;
  float2 A2[kStates], h[kStates], total = f2(0.0f);
#pragma unroll
  for (int q = 0; q < kStates; ++q) h[q] = A2[q] = f2(0.0f);
  const int c_scan = grp * g.Dg + 2 * pair;
  const bool second_scan = 2 * pair + 1 < g.Dg;
  const int64_t place = g.slots ? (int64_t)g.slots[b] : (int64_t)b;
  const bool has_place = place >= 0 && place < g.num_slots;
  if (scans) {
    load_states(g.A + (int64_t)c_scan * g.N, g.N, pl * kStates, second_scan, A2);
#pragma unroll
    for (int q = 0; q < kStates; ++q) A2[q] = mul2(A2[q], f2(kLog2E));
    if (MODE == kEnds && span == 0) {
      // the state before the first token, where the last span's end would be: the
      // kernel after this one may write it while its warps start from it
      float2 h0[kStates] = {f2(0.0f), f2(0.0f), f2(0.0f), f2(0.0f)};
      if (g.state_in && has_place)
        load_states(g.state_in + (place * g.D + c_scan) * g.N, g.N, pl * kStates, second_scan, h0);
      store_own(g.ends + ((int64_t)(g.spans - 1) * own_all + own) * 2 * kStates, h0);
    }
    if (MODE == kFull) {
      if (g.spans > 1) {
        load_own(g.ends + ((int64_t)(g.spans - 1) * own_all + own) * 2 * kStates, h);
#pragma unroll 4
        for (int i = 0; i < span; ++i) {
          float2 e[kStates];
          load_own(g.ends + ((int64_t)i * own_all + own) * 2 * kStates, e);
          const float2 s = g.sums[((int64_t)i * g.B * g.G + rest) * g.pairs + pair];
#pragma unroll
          for (int q = 0; q < kStates; ++q) h[q] = fma2(ex2(mul2(s, A2[q])), h[q], e[q]);
        }
      } else if (g.state_in && has_place) {
        load_states(g.state_in + (place * g.D + c_scan) * g.N, g.N, pl * kStates, second_scan, h);
      }
    }
  }

  // the thread's channel pair where tokens are loaded and stored
  const int pr = lane % PW, row = lane / PW;
  const bool loads = row < R && pair0 + pr < g.pairs;
  const int c = grp * g.Dg + 2 * (pair0 + pr);
  const bool second = 2 * (pair0 + pr) + 1 < g.Dg, pairs_ok = g.pair_ok, gate = MODE != kEnds && g.z.data;
  float2 bias = f2(0.0f), skip = f2(0.0f);
  if (loads) {
    if (g.bias) bias = make_float2(g.bias[c], second ? g.bias[c + 1] : 0.0f);
    if (MODE == kFull && g.D_skip) skip = make_float2(g.D_skip[c], second ? g.D_skip[c + 1] : 0.0f);
  }
  const Seq& in = MODE == kBack ? g.gy : g.u;
  const T* const pu = static_cast<const T*>(in.data) + b * in.sb + c;
  const T* const pd = static_cast<const T*>(g.delta.data) + b * g.delta.sb + c;
  const T* const pz = static_cast<const T*>(g.z.data) + b * g.z.sb + c;
  T* const py = static_cast<T*>(g.y.data) + b * g.y.sb + c;
  Raw<T> raw_u[kUnits], raw_d[kUnits], raw_z[kUnits];
  const int stop = last < len ? last : len;  // tokens that exist
  auto fetch = [&](int t0) {
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
      const int tok = row + k * R, now = t0 + tok;
      raw_u[k].clear();
      raw_d[k].clear();
      raw_z[k].clear();
      if (loads && tok < kTile && now < stop) {
        raw_u[k].load(pu + now * in.st, pairs_ok, second);
        raw_d[k].load(pd + now * g.delta.st, pairs_ok, second);
        if (gate) raw_z[k].load(pz + now * g.z.st, pairs_ok, second);
      }
    }
  };

  const int tiles = stop > first ? (stop - first + kTile - 1) / kTile : 0;
  float* ckpt = nullptr;
  const int64_t ckpt_step = (int64_t)g.G * g.pairs * P * 2 * kStates;
  if (MODE == kFull && g.ckpt && scans)
    ckpt = g.ckpt + ((int64_t)b * ((g.T + kTile - 1) / kTile) + first / kTile) * ckpt_step +
           (((int64_t)grp * g.pairs + pair) * P + pl) * 2 * kStates;
  if (tiles) fetch(MODE == kBack ? first + (tiles - 1) * kTile : first);
  for (int tile = 0; tile < tiles; ++tile) {
    const int t0 = first + (MODE == kBack ? tiles - 1 - tile : tile) * kTile;
    if (MODE != kBack) load_tile<T>(g, g.Bm, Bd, P, b, grp, t0, stop, lane);
    if (MODE != kEnds) load_tile<T>(g, g.Cm, Cd, P, b, grp, t0, stop, lane);
    Raw<T> now_u[kUnits], now_z[kUnits];
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
      const int tok = row + k * R;
      now_u[k] = raw_u[k];
      now_z[k] = raw_z[k];
      if (loads && tok < kTile) {
        float2 s = f2(0.0f), x = f2(0.0f);
        if (t0 + tok < stop) {
          s = step_of(add2(raw_d[k].get(), bias), g.softplus);
          x = raw_u[k].get();
          if (MODE == kBack) {
            if (gate) x = mul2(x, mul2(raw_z[k].get(), sigmoid<T>(raw_z[k].get())));
          } else {
            x = mul2(s, x);
          }
          if (!second) s.y = x.y = 0.0f;
        }
        sx[tok * PW + pr] = make_float4(s.x, s.y, x.x, x.y);
      }
    }
    __syncwarp();
    if (tile + 1 < tiles) fetch(MODE == kBack ? t0 - kTile : t0 + kTile);
    if (scans) {
      if (MODE == kFull && ckpt) {
        store_own(ckpt, h);
        ckpt += ckpt_step;
      }
#pragma unroll
      for (int i = 0; i < kTile; ++i) {
        const int tok = MODE == kBack ? kTile - 1 - i : i;
        const float4 v = sx[tok * PW + pc];
        const float2 s = make_float2(v.x, v.y), x = make_float2(v.z, v.w);
        float2 bc[kStates];
        load_own(reinterpret_cast<const float*>((MODE == kBack ? Cd : Bd) + (tok * P + pl) * kStates), bc);
#pragma unroll
        for (int q = 0; q < kStates; ++q) {
          const float2 a = ex2(mul2(s, A2[q]));
          if (MODE == kBack) h[q] = mul2(a, fma2(x, bc[q], h[q]));
          else h[q] = fma2(a, h[q], mul2(x, bc[q]));
        }
        if (MODE == kFull) {
          load_own(reinterpret_cast<const float*>(Cd + (tok * P + pl) * kStates), bc);
          float2 y = mul2(bc[0], h[0]);
#pragma unroll
          for (int q = 1; q < kStates; ++q) y = fma2(bc[q], h[q], y);
          yp[tok * 32 + lane] = y;
        } else {
          total = add2(total, s);
        }
      }
    }
    __syncwarp();
    if (MODE == kFull) {
#pragma unroll
      for (int k = 0; k < kUnits; ++k) {
        const int tok = row + k * R, now = t0 + tok;
        if (loads && tok < kTile && now < last) {
          float2 y = f2(0.0f);
          if (now < stop) {
            y = sum_parts<PT>(yp + tok * 32 + pr * P, P);
            y = fma2(skip, now_u[k].get(), y);
            if (gate) {
              const float2 z = now_z[k].get();
              y = mul2(y, mul2(z, sigmoid<T>(z)));
            }
          }
          put_pair(py + now * g.y.st, y, pairs_ok, second);
        }
      }
    }
  }
  if (MODE == kFull) {
    // places past the sequence's end
    if (loads)
      for (int now = first + tiles * kTile + row; now < last; now += R)
        put_pair(py + now * g.y.st, f2(0.0f), pairs_ok, second);
    if (scans && g.state_out && has_place && span == g.spans - 1)
      store_states(g.state_out + (place * g.D + c_scan) * g.N, g.N, pl * kStates, second_scan, h);
  } else if (scans) {
    store_own(g.ends + ((int64_t)span * own_all + own) * 2 * kStates, h);
    if (pl == 0) g.sums[((int64_t)span * g.B * g.G + rest) * g.pairs + pair] = total;
  }
}

template <typename T, int MODE>
cudaError_t launch_mode(const Args& g, int spans, cudaStream_t st) {
  const int64_t blocks = (int64_t)g.B * g.G * ceil_div(g.pairs, 32 / g.P);
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)blocks, (unsigned)spans);
  const size_t smem = fwd_smem(g.P, MODE);
  if (g.P == 4) return launch_pdl(scan_fwd<T, MODE, 4>, grid, dim3(32), smem, st, g);
  return launch_pdl(scan_fwd<T, MODE, 0>, grid, dim3(32), smem, st, g);
}

template <typename T>
cudaError_t launch_fwd(const Args& g, cudaStream_t st) {
  if (g.spans > 1) {
    const cudaError_t e = launch_mode<T, kEnds>(g, g.spans - 1, st);
    if (e != cudaSuccess) return e;
  }
  return launch_mode<T, kFull>(g, g.spans, st);
}

cudaError_t launch_back_ends(const Args& g, int dtype, cudaStream_t st) {
  if (dtype == SNN_F32) return launch_mode<float, kBack>(g, g.spans - 1, st);
  if (dtype == SNN_BF16) return launch_mode<__nv_bfloat16, kBack>(g, g.spans - 1, st);
  return launch_mode<__half, kBack>(g, g.spans - 1, st);
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
  return snn::ceil_div(d.T, kTile) * g.B * g.G * g.pairs * g.P * 2 * kStates;
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
  const Plan plan = fwd_plan(g);
  g.spans = plan.spans;
  g.span = plan.span;
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
  g.sums = reinterpret_cast<float2*>(w + ends_bytes(g, plan.spans));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = desc->dtype == SNN_F32    ? launch_fwd<float>(g, st)
                        : desc->dtype == SNN_BF16 ? launch_fwd<__nv_bfloat16>(g, st)
                                                  : launch_fwd<__half>(g, st);
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

}  // extern "C"
