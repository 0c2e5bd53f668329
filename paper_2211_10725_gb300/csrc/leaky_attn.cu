// Leaky attention over whole sequences: entry points and kernels.
//   S_t = beta S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t
// and its gradients, which are the same recurrence with the tensors' roles
// changed (see leaky_attn.cuh).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <type_traits>

#include "launch.cuh"
#include "leaky_attn.cuh"
#include "leaky_attn_chunks.cuh"
#include "leaky_attn_host.cuh"
#include "scan_host.cuh"

namespace snn {
namespace attn {

// A shared head's gradients: out[b, t, hk, :] = sum over the group's query
// heads, in head order, of their fp32 shares part[b, t, h, :], rounded once.
// blockIdx.y picks the gradient (of k or of v).  The shares stay fp32 so that a
// shared head's gradient is rounded once (3 x 777 tokens, 12 heads on 4: 8 us from a
// cold cache, 62 for the whole backward).
struct SumArgs {
  const float* part[2];
  Tensor out[2];
  int D[2];
  int Hk, G;
  int64_t T, rows;  // rows: (b, t, hk)
};

template <typename T>
__global__ void __launch_bounds__(256) sum_group(const SumArgs g) {
  grid_dep_wait();
  const int which = blockIdx.y, D = g.D[which], d8 = D / 8;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= g.rows * d8) return;
  const int d = (int)(i % d8) * 8;
  const int64_t row = i / d8, bt = row / g.Hk;
  const int hk = (int)(row % g.Hk);
  const float* p = g.part[which] + row * g.G * D + d;
  float s[8];
  Elem<float>::load8(p, s);
  for (int j = 1; j < g.G; ++j) {
    float v[8];
    Elem<float>::load8(p + (int64_t)j * D, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += v[e];
  }
  const Tensor& o = g.out[which];
  Elem<T>::store8(static_cast<T*>(o.data) + (bt / g.T) * o.sb + (bt % g.T) * o.st + hk * o.sh + d, s);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

// How a run over `heads` heads (of all its roles) cuts T tokens into segments:
// the count that should end soonest, from the times (us) of a chunk in a block
// alone on its SM and in one of a full SM, and of a block's start:
//   128 x 128 tiles, two blocks on an SM: attn_chunks 2.6 alone, 3.65 beside
//   another (64 chunks in one and two blocks on every SM: 172 and 240);
//   attn_segments 1.05 and 1.8;
//   64 x 64 tiles: attn_chunks, three blocks on an SM, 2.0 and 3.0 (64 chunks
//   in one, two and three blocks on every SM: 131, 171 and 197);
//   attn_segments, four blocks, 0.65 and 1.6;
//   tiles of both widths, two blocks on an SM: between these (64 x 128: 136 and
//   189; 128 x 64: 146 and 205).
// A function of the shapes alone, so that a shape always sums in the same
// order.
struct Plan {
  int da = 64, dc = 64;  // the tile: widths of a/b and of c/out, 64 or 128
  int nseg = 1, seg_tokens = kChunk;
  int64_t heads = 0;
  double time = 0.0;
  size_t bytes() const {  // of the segments' states
    return nseg == 1 ? 0 : (size_t)heads * nseg * da * dc * sizeof(float);
  }
};
constexpr int kMaxSeg = 64;
constexpr int kSummed = 4;  // segments whose states the blocks sum themselves
constexpr int kSms = 152;
inline int tile(int64_t D) { return D <= 64 ? 64 : 128; }

// Time of `blocks` blocks of `per` chunks, at most per_sm on an SM.
double wave_time(int64_t blocks, int64_t per, int per_sm, double alone, double full) {
  constexpr double kStart = 5.0;
  const int64_t slots = (int64_t)kSms * per_sm, rest = blocks % slots;
  const double on_sm = (double)ceil_div(rest, kSms);
  const double chunk = alone + (full - alone) * (on_sm - 1.0) / (per_sm - 1);
  return (double)(blocks / slots) * (kStart + full * per) + (rest ? kStart + chunk * per : 0.0);
}

Plan plan(int64_t T, int64_t heads, int da, int dc) {
  Plan best;
  best.da = da;
  best.dc = dc;
  best.heads = heads;
  const int64_t chunks = ceil_div(T, kChunk);
  const int kind = (da + dc) / 64 - 2;  // 0: 64 x 64, 1: both, 2: 128 x 128
  const int per_sm = kind == 0 ? 3 : 2, seg_per_sm = kind == 0 ? 4 : 2;
  constexpr double kAlone[3] = {2.0, 2.1, 2.6}, kFull[3] = {3.0, 3.0, 3.65};
  constexpr double kSegAlone[3] = {0.65, 0.85, 1.05}, kSegFull[3] = {1.6, 1.6, 1.8};
  constexpr double kLaunch = 3.0, kScan = 2.0;
  for (int64_t s = 1; s <= kMaxSeg && s <= chunks; ++s) {
    const int64_t per = ceil_div(chunks, s), n = ceil_div(chunks, per);
    double t = wave_time(heads * n, per, per_sm, kAlone[kind], kFull[kind]);
    if (n > 1)
      t += kLaunch + wave_time(heads * (n - 1), per, seg_per_sm, kSegAlone[kind], kSegFull[kind]);
    if (n > 1) t += n > kSummed ? kScan + 0.1 * n : 0.8 * n;
    if (s == 1 || t < best.time) {
      best.time = t;
      best.nseg = (int)n;
      best.seg_tokens = (int)(per * kChunk);
    }
  }
  return best;
}

Plan plan_fwd(const snn_attn_desc* d) { return plan(d->T, d->B * d->H, tile(d->Dk), tile(d->Dv)); }

// The backward's three roles: in one launch where their tiles are the same.
// Where Dk and Dv differ in tile, grad_q and grad_k have the widths the other way
// round from grad_v: in two launches, or, where that ends sooner, in one with
// 128 x 128 tiles, whose blocks are longer but fill the SMs at once. 64 x 128,
// one launch against two: 92 us and 123 (6 x 1500 tokens, 16 heads), 17 and 28
// (300 tokens, 8 heads); 350 and 296 (8 x 2048, 32 heads), 323 and 287
// (32 x 512, 32 heads).
struct BwdPlan {
  bool one = true;
  Plan first, last;  // first: all three, or grad_q and grad_k; last: grad_v
  size_t bytes() const { return first.bytes() + (one ? 0 : last.bytes()); }
};
BwdPlan plan_bwd(const snn_attn_desc* d) {
  const int64_t heads = d->B * d->H;
  const int tk = tile(d->Dk), tv = tile(d->Dv);
  BwdPlan p;
  p.first = plan(d->T, 3 * heads, tk > tv ? tk : tv, tk > tv ? tk : tv);
  if (tk == tv) return p;
  const Plan two = plan(d->T, 2 * heads, tv, tk);
  p.last = plan(d->T, heads, tk, tv);
  if (two.time + p.last.time < p.first.time) {
    p.one = false;
    p.first = two;
  }
  return p;
}

// Map of a [B, T, heads, D] tensor read or written as boxes of 64 tokens x 128
// bytes (64 16-bit elements, or 32 fp32 ones) of one head; tokens past T and
// elements past D read as zero and are not written.
bool make_map_bthd(CUtensorMap* map, const Tensor& x, const Args& g, int heads, int D,
                   CUtensorMapDataType type) {
  auto fn = gemm::encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)g.T, (cuuint64_t)heads, (cuuint64_t)g.B};
  // the stride of an extent of 1 is never stepped over: any valid value
  const int size = type == CU_TENSOR_MAP_DATA_TYPE_FLOAT32 ? 4 : 2;
  auto bytes = [&](int64_t extent, int64_t stride) { return (cuuint64_t)(extent == 1 ? 16 : size * stride); };
  const cuuint64_t strides[3] = {bytes(g.T, x.st), bytes(heads, x.sh), bytes(g.B, x.sb)};
  const cuuint32_t box[4] = {128u / size, (cuuint32_t)kChunk, 1u, 1u};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, type, 4, x.data, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DA, int DC>
cudaError_t launch_tile(ChunkArgs& p, cudaStream_t st) {
  using C = Cfg<DA, DC>;
  const cudaError_t e = ensure_smem((const void*)attn_chunks<T, DA, DC>, C::kSmem);
  if (e != cudaSuccess) return e;
  const int64_t blocks = (int64_t)p.g.B * p.g.H * p.nseg * p.g.nroles;
  if (p.nseg > 1) {
    // a third part of the decayed values only where a bf16 state is an output
    bool third = false;
    for (int i = 0; i < p.g.nroles; ++i)
      third = third || (p.g.role[i].s_out && std::is_same<T, __nv_bfloat16>::value);
    const size_t smem = C::kSegSmem + (third ? C::kCBytes : 0);
    // up to four states are summed sooner by the segments themselves (2x4096
    // tokens of 32 heads, four segments: 97 us, 102 with the scan)
    p.scanned = p.nseg > kSummed;
    cudaError_t es = ensure_smem((const void*)attn_segments<T, DA, DC>, smem);
    if (es == cudaSuccess)
      es = launch_pdl(attn_segments<T, DA, DC>, dim3((unsigned)blocks), dim3(C::kThreads), smem, st, p);
    if (es == cudaSuccess && p.scanned) {
      const int64_t heads = (int64_t)p.g.B * p.g.H * p.g.nroles;
      es = launch_pdl(attn_segment_scan, dim3((unsigned)(heads * (DA * DC / (4 * kScanThreads)))),
                      dim3(kScanThreads), 0, st, p, DA * DC);
    }
    if (es != cudaSuccess) return es;
  }
  return launch_pdl(attn_chunks<T, DA, DC>, dim3((unsigned)blocks), dim3(C::kThreads), C::kSmem, st, p);
}

template <typename T>
cudaError_t launch(const Args& g, const Plan& pl, float* seg_state, cudaStream_t st) {
  ChunkArgs p = {};
  p.g = g;
  p.nseg = pl.nseg;
  p.seg_tokens = pl.seg_tokens;
  p.seg_state = seg_state;
  constexpr CUtensorMapDataType kType = std::is_same<T, __nv_bfloat16>::value
                                            ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                            : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  for (int i = 0; i < g.nroles && g.T > 0; ++i) {
    const Role& r = g.role[i];
    if (!make_map_bthd(&p.map[i].a, r.a, g, g.H / r.a.group, r.Da, kType) ||
        !make_map_bthd(&p.map[i].b, r.b, g, g.H / r.b.group, r.Da, kType) ||
        !make_map_bthd(&p.map[i].c, r.c, g, g.H / r.c.group, r.Dc, kType) ||
        !make_map_bthd(&p.map[i].out, r.out, g, g.H / r.out.group, r.Dc,
                       r.out_f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : kType))
      return cudaErrorInvalidValue;
  }
  if (pl.da == 64) return pl.dc == 64 ? launch_tile<T, 64, 64>(p, st) : launch_tile<T, 64, 128>(p, st);
  return pl.dc == 64 ? launch_tile<T, 128, 64>(p, st) : launch_tile<T, 128, 128>(p, st);
}

cudaError_t launch(const snn_attn_desc* d, const Args& g, const Plan& pl, float* seg_state, cudaStream_t st) {
  return d->dtype == SNN_BF16 ? launch<__nv_bfloat16>(g, pl, seg_state, st)
                              : launch<__half>(g, pl, seg_state, st);
}

template <typename T>
cudaError_t launch_sum(const SumArgs& g, cudaStream_t st) {
  const int64_t n8 = g.rows * ((g.D[0] > g.D[1] ? g.D[0] : g.D[1]) / 8);
  return launch_pdl(sum_group<T>, dim3((unsigned)((n8 + 255) / 256), 2), dim3(256), 0, st, g);
}

size_t share_bytes(const snn_attn_desc* d, int64_t D) {
  return d->H == d->Hk ? 0 : round256((size_t)(d->B * d->T * d->H * D) * sizeof(float));
}

Args base_args(const snn_attn_desc* d, const float* beta, const int32_t* seq_lens, void* ws) {
  Args g;
  g.B = (int)d->B;
  g.T = (int)d->T;
  g.H = (int)d->H;
  g.Dk = (int)d->Dk;
  g.Dv = (int)d->Dv;
  g.scale = d->scale;
  g.beta = beta;
  g.seq_lens = seq_lens;
  g.status = static_cast<int*>(ws);
  return g;
}

}  // namespace attn
}  // namespace snn

using namespace snn::attn;

extern "C" {

size_t snn_attn_desc_size(void) { return sizeof(snn_attn_desc); }

size_t snn_leaky_attn_workspace_bytes(const snn_attn_desc* desc, int backward) {
  if (check_desc(desc) != SNN_OK) return 0;
  const size_t fwd = plan_fwd(desc).bytes();
  if (!backward) return 256 + fwd;
  const size_t bwd =
      plan_bwd(desc).bytes() + share_bytes(desc, desc->Dk) + share_bytes(desc, desc->Dv);
  return 256 + (fwd > bwd ? fwd : bwd);
}

snn_status_t snn_leaky_attn_fwd(const snn_attn_desc* desc, const snn_bthd* q, const snn_bthd* k,
                                const snn_bthd* v, const float* beta, const int32_t* seq_lens,
                                const float* state_in, float* state_out, const int32_t* slots,
                                int64_t num_slots, const snn_bthd* o, void* ws, size_t ws_bytes,
                                snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  const snn_bthd* x[4] = {q, k, v, o};
  const int64_t heads[4] = {desc->H, desc->Hk, desc->Hk, desc->H};
  for (int i = 0; i < 4; ++i)
    if ((s = check_tensor(desc, x[i], heads[i])) != SNN_OK) return s;
  if (!beta || (slots && num_slots < 0)) return SNN_ERR_INVALID_ARG;
  const void* ptrs[6] = {beta, seq_lens, state_in, state_out, slots, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  if (!ws || ws_bytes < snn_leaky_attn_workspace_bytes(desc, 0)) return SNN_ERR_WORKSPACE;
  if (desc->B == 0) return SNN_OK;
  const int G = (int)(desc->H / desc->Hk);
  Args g = base_args(desc, beta, seq_lens, ws);
  g.slots = slots;
  g.num_slots = slots ? num_slots : desc->B;
  g.nroles = 1;
  snn::attn::Role& r = g.role[0];
  r.a = tensor(q, 1);
  r.b = tensor(k, G);
  r.c = tensor(v, G);
  r.out = tensor(o, 1);
  r.Da = g.Dk;
  r.Dc = g.Dv;
  r.s_in = state_in;
  r.s_out = state_out;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  float* seg_state = reinterpret_cast<float*>(static_cast<unsigned char*>(ws) + 256);
  const cudaError_t e = launch(desc, g, plan_fwd(desc), seg_state, st);
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

snn_status_t snn_leaky_attn_bwd(const snn_attn_desc* desc, const snn_bthd* q, const snn_bthd* k,
                                const snn_bthd* v, const float* beta, const int32_t* seq_lens,
                                const float* state_in, const snn_bthd* grad_o,
                                const float* grad_state_out, const snn_bthd* grad_q,
                                const snn_bthd* grad_k, const snn_bthd* grad_v,
                                float* grad_state_in, void* ws, size_t ws_bytes,
                                snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  // the gradient of the end state is divided by it
  if (!std::isnormal(desc->scale) || !std::isnormal(1.0f / desc->scale)) return SNN_ERR_INVALID_ARG;
  const snn_bthd* x[7] = {q, k, v, grad_o, grad_q, grad_k, grad_v};
  const int64_t heads[7] = {desc->H, desc->Hk, desc->Hk, desc->H, desc->H, desc->Hk, desc->Hk};
  for (int i = 0; i < 7; ++i)
    if ((s = check_tensor(desc, x[i], heads[i])) != SNN_OK) return s;
  if (!beta) return SNN_ERR_INVALID_ARG;
  // one role writes the one while the others read the other two
  if (grad_state_in && (grad_state_in == grad_state_out || grad_state_in == state_in))
    return SNN_ERR_INVALID_ARG;
  const void* ptrs[6] = {beta, seq_lens, state_in, grad_state_out, grad_state_in, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  if (!ws || ws_bytes < snn_leaky_attn_workspace_bytes(desc, 1)) return SNN_ERR_WORKSPACE;
  if (desc->B == 0) return SNN_OK;
  const int G = (int)(desc->H / desc->Hk);
  Args g = base_args(desc, beta, seq_lens, ws);
  g.num_slots = desc->B;
  g.nroles = 3;
  unsigned char* at = static_cast<unsigned char*>(ws) + 256;
  float* seg_state = reinterpret_cast<float*>(at);
  const BwdPlan pl = plan_bwd(desc);
  at += pl.bytes();
  float* share_k = reinterpret_cast<float*>(at);
  float* share_v = reinterpret_cast<float*>(at + share_bytes(desc, desc->Dk));
  auto share = [&](float* p, int64_t D) {
    Tensor t;
    t.data = p;
    t.sh = D;
    t.st = desc->H * D;
    t.sb = desc->T * t.st;
    return t;
  };
  snn::attn::Role& rq = g.role[0];
  rq.a = tensor(grad_o, 1);
  rq.b = tensor(v, G);
  rq.c = tensor(k, G);
  rq.out = tensor(grad_q, 1);
  rq.Da = g.Dv;
  rq.Dc = g.Dk;
  rq.s_in = state_in;
  rq.s_trans = 1;
  snn::attn::Role& rk = g.role[1];
  rk.a = tensor(v, G);
  rk.b = tensor(grad_o, 1);
  rk.c = tensor(q, 1);
  rk.out = G == 1 ? tensor(grad_k, 1) : share(share_k, desc->Dk);
  rk.Da = g.Dv;
  rk.Dc = g.Dk;
  rk.rev = 1;
  rk.s_in = grad_state_out;
  rk.s_trans = 1;
  snn::attn::Role& rv = g.role[2];
  rv.a = tensor(k, G);
  rv.b = tensor(q, 1);
  rv.c = tensor(grad_o, 1);
  rv.out = G == 1 ? tensor(grad_v, 1) : share(share_v, desc->Dv);
  rv.Da = g.Dk;
  rv.Dc = g.Dv;
  rv.rev = 1;
  rv.s_in = grad_state_out;
  rv.s_out = grad_state_in;
  rv.out_f32 = rk.out_f32 = G > 1;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (pl.one) {
    e = launch(desc, g, pl.first, seg_state, st);
  } else {
    Args gv = g;
    gv.role[0] = rv;
    gv.nroles = 1;
    g.nroles = 2;
    e = launch(desc, g, pl.first, seg_state, st);
    if (e == cudaSuccess)
      e = launch(desc, gv, pl.last, seg_state + pl.first.bytes() / sizeof(float), st);
  }
  if (e == cudaSuccess && G > 1 && desc->T > 0) {
    const SumArgs sum{{share_k, share_v},  {tensor(grad_k, 1), tensor(grad_v, 1)}, {g.Dk, g.Dv},
                      (int)desc->Hk,       G,
                      desc->T,             desc->B * desc->T * desc->Hk};
    e = desc->dtype == SNN_BF16 ? launch_sum<__nv_bfloat16>(sum, st) : launch_sum<__half>(sum, st);
  }
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

}  // extern "C"
