// Leaky attention in chunks on the tensor cores.
//
// With E the state a chunk starts from, already decayed to its first token,
// the recurrence over n <= 64 tokens is four products (i, j count tokens in
// the direction of time of the role, see leaky_attn.cuh):
//   scores  s_ij = a_i . b_j                                [64 x 64]
//   inter   (scale beta^i a_i) E                            [64 x Dc]
//   intra   + sum_{j <= i} (scale beta^(i-j) s_ij) c_j      [64 x Dc], same accumulator
//   update  E <- beta^n E + sum_j b_j (beta^(n-j) c_j)^T    [Da x Dc]
// A block walks the chunks of one head in order with E in fp32 registers, so
// every token is read once and the state never leaves the SM.  Operands land
// by TMA as 64-token, 64-element boxes (128-byte swizzle); the same box of b
// is the K-major operand of the scores and the MN-major one of the update.
// Per chunk one thread issues the MMAs in two groups with the block's work
// between: the decayed scores, queries and values go back to shared memory as
// 16-bit operands; then the state is updated from its accumulator while the
// intra product runs, and the output leaves by TMA.  Two blocks (128-wide
// heads) or four (64-wide) share an SM and fill each other's waits; 64-token
// chunks are what lets two 112 KB working sets fit.
//
// Roundings to 16 bits: the operands (decayed scores, queries, values and the
// state's copy) and the output.  The state itself is a sum of fp32
// accumulators; where it is an output, the decayed values are split into two
// 16-bit parts and multiplied twice, so it keeps 16 bits or more per term.
// The state's copy is bf16 even for fp16 tensors, for its range.
//
// Few heads and many tokens: the tokens are cut into segments, a first launch
// finds each segment's own contribution to the state (update products only),
// and each segment then starts from the decayed sum of those before it.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "launch.cuh"
#include "leaky_attn.cuh"
#include "snn_device.cuh"
#include "tcgen05.cuh"

namespace snn {
namespace attn {

constexpr int kChunk = 64;
constexpr int kBoxBytes = kChunk * 128;  // 64 tokens x 64 16-bit elements
constexpr uint64_t kWaitNs = 2000000000ull;

struct RoleMaps {
  CUtensorMap a, b, c, out;
};

struct ChunkArgs {
  Args g;
  RoleMaps map[kMaxRoles];
  int nseg;             // segments of a sequence
  int seg_tokens;       // tokens of a segment, a multiple of kChunk
  int states_only;      // the first launch of a segmented run
  float* seg_state;     // [role][B*H][nseg] states in fragment order
};

template <int DA, int DC>
struct Cfg {
  static constexpr int kThreads = (DA == 128 || DC == 128) ? 256 : 128;
  static constexpr int kHalves = kThreads / 128;  // column halves of an accumulator
  static constexpr int kCols = DC / kHalves;      // columns of c/out a warp covers
  static constexpr int kRowHalves = DA / 64;      // 16-lane halves of the state accumulator
  static constexpr int kState = kRowHalves * kCols / 2;  // state floats of a thread
  static constexpr int kABytes = kChunk * DA * 2;
  static constexpr int kCBytes = kChunk * DC * 2;
  static constexpr int kEBytes = DA * DC * 2;
  static constexpr int kOutBytes = kCBytes;       // >= the 8 KB of the decayed scores
  static constexpr int kTail = 1024;              // barriers, tables
  static constexpr size_t kSmem = 2 * kABytes + 2 * kCBytes + kEBytes + kOutBytes + kTail;
  static constexpr uint32_t kTmemCols = 2 * DC;   // scores/output, state update
  static constexpr int kBlocksPerSm = kThreads == 128 ? 4 : 2;
};

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z,
                                            int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
          smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
      : "memory");
}

__device__ __forceinline__ void tma_store_4d(const CUtensorMap* map, const void* src, int x, int y,
                                             int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(
          reinterpret_cast<uint64_t>(map)),
      "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}

__device__ __forceinline__ void bulk_wait_read_all() {
  asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}

// 16 lanes x 32 columns of TMEM: register 4k + 2r + c of lane l holds row
// l/4 + 8r, column 8k + 2(l%4) + c.
__device__ __forceinline__ void tmem_ld_rows16(uint32_t taddr, float v[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, "
      "%12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// MN-major descriptor whose next 64 elements along MN are box_bytes on.
__device__ __forceinline__ uint64_t sdesc_mn(const void* tile, uint32_t box_bytes) {
  uint64_t d = gemm::sdesc_sw128(tile);
  d &= ~(uint64_t(0x3FFF) << 16);
  return d | (uint64_t)(box_bytes >> 4) << 16;
}

template <typename T>
__host__ __device__ constexpr uint32_t idesc(int m, int n, bool a_mn, bool b_mn) {
  const uint32_t d = gemm::idesc_bf16(m, n, a_mn, b_mn);
  return std::is_same<T, __half>::value ? d & ~((1u << 7) | (1u << 10)) : d;  // format 0: fp16
}

// Wait of every thread of the block; the warp is whole again afterwards, as
// the tensor-memory loads that follow need.
__device__ __forceinline__ int wait_all(uint64_t* bar, uint32_t parity) {
  const int fail = !gemm::mbar_wait_poll(bar, parity, kWaitNs);
  __syncwarp();
  return fail;
}

template <typename T, int DA, int DC>
__global__ void __launch_bounds__(Cfg<DA, DC>::kThreads, Cfg<DA, DC>::kBlocksPerSm)
    attn_chunks(const __grid_constant__ ChunkArgs p) {
  using C = Cfg<DA, DC>;
  using BF = __nv_bfloat16;
  constexpr int NT = C::kThreads;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* sA = smem;
  unsigned char* sB = sA + C::kABytes;
  unsigned char* sC = sB + C::kABytes;
  unsigned char* sW = sC + C::kCBytes;   // decayed values
  unsigned char* sE = sW + C::kCBytes;   // the state's copy
  unsigned char* sP = sE + C::kEBytes;   // decayed scores, then the output
  uint64_t* bar = reinterpret_cast<uint64_t*>(sP + C::kOutBytes);
  uint64_t *bar_ab = bar, *bar_c = bar + 1, *bar_s = bar + 2, *bar_u = bar + 3, *bar_o = bar + 4,
           *bar_l = bar + 5;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + 6);
  float* pw = reinterpret_cast<float*>(bar + 8);  // beta^n, n = 0 .. 64
  float* ptab = pw + 68;                          // scale * beta^n, n = 0 .. 63

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int quad = warp & 3, half = warp >> 2;
  const Args& g = p.g;
  const int role = blockIdx.x % g.nroles;
  const int seg = (blockIdx.x / g.nroles) % p.nseg;
  const int row = blockIdx.x / (g.nroles * p.nseg);
  const int b = row / g.H, h = row % g.H;
  const Role& r = g.role[role];
  const RoleMaps& maps = p.map[role];
  const int rev = r.rev;

  if (tid == 0) {
    for (int i = 0; i < 6; ++i) mbar_init(&bar[i], 1);
    fence_barrier_init();
  }
  __syncwarp();
  if (warp == 0) gemm::tmem_alloc(tmem_slot, C::kTmemCols);
  gemm::tc_fence_before();
  __syncthreads();
  gemm::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_dep_wait();

  const int len = seq_len(g, b);
  const int t_begin = seg * p.seg_tokens;
  const int t_end = min(g.T, t_begin + p.seg_tokens);
  const int last_seg = len > 0 ? (len - 1) / p.seg_tokens : 0;
  const int order = rev ? last_seg - seg : seg;  // place of this segment in time
  const int n_tok = max(0, min(len, t_end) - t_begin);
  int n_chunks = (n_tok + kChunk - 1) / kChunk;
  if (p.states_only && order >= last_seg) n_chunks = 0;  // nothing starts after this one
  const bool active = seg <= last_seg;
  const bool ends = !p.states_only && r.s_out && (rev ? seg == 0 : seg == last_seg);

  // the first loads
  auto chunk_start = [&](int it) { return t_begin + kChunk * (rev ? n_chunks - 1 - it : it); };
  auto load_ab = [&](int it) {
    const int t0 = chunk_start(it);
    mbar_arrive_expect_tx(bar_ab, (p.states_only ? 1 : 2) * C::kABytes);
#pragma unroll
    for (int x = 0; x < DA / 64; ++x) {
      if (!p.states_only)
        tma_load_4d(sA + x * kBoxBytes, &maps.a, 64 * x, t0, h / r.a.group, b, bar_ab);
      tma_load_4d(sB + x * kBoxBytes, &maps.b, 64 * x, t0, h / r.b.group, b, bar_ab);
    }
  };
  auto load_c = [&](int it) {
    mbar_arrive_expect_tx(bar_c, C::kCBytes);
#pragma unroll
    for (int x = 0; x < DC / 64; ++x)
      tma_load_4d(sC + x * kBoxBytes, &maps.c, 64 * x, chunk_start(it), h / r.c.group, b, bar_c);
  };
  if (tid == 0 && n_chunks > 0) {
    load_ab(0);
    load_c(0);
  }

  // powers of the decay, in fp64 by squaring: each one correctly rounded
  const double beta = (double)g.beta[h];
  auto power = [&](int n) {
    double v = 1.0, s = beta;
    for (; n > 0; n >>= 1, s *= s)
      if (n & 1) v *= s;
    return v;
  };
  if (tid <= kChunk) {
    const float v = (float)power(tid);
    pw[tid] = v;
    if (tid < kChunk) ptab[tid] = v * g.scale;
  }
  __syncthreads();

  // this thread's part of the state: rows erow + 16*rh (+8), columns ecol + 8k (+1)
  const int erow = (C::kRowHalves == 2 ? 32 : 16) * quad + (lane >> 2);
  const int ecol = half * C::kCols + 2 * (lane & 3);
  float E[C::kState];
  const int64_t so = (r.s_in || r.s_out) ? state_offset(g, b, h) : -1;
  const int64_t s_row = r.s_trans ? 1 : g.Dv, s_col = r.s_trans ? g.Dv : 1;
  auto each_state = [&](auto f) {  // f(index, row, column) over the thread's part
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh)
#pragma unroll
      for (int k = 0; k < C::kCols / 8; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          f((rh * (C::kCols / 8) + k) * 4 + e, erow + 16 * rh + 8 * (e >> 1), ecol + 8 * k + (e & 1));
  };
  const size_t seg_stride = (size_t)DA * DC;
  float* const seg0 = p.seg_state + ((size_t)role * g.B * g.H + row) * p.nseg * seg_stride;
  if (order == 0 && (p.nseg == 1 || p.states_only)) {
    const float f = rev ? 1.0f / g.scale : (len > 0 ? pw[1] : 1.0f);
    each_state([&](int i, int y, int x) {
      E[i] = r.s_in && so >= 0 && y < r.Da && x < r.Dc ? f * r.s_in[so + y * s_row + x * s_col] : 0.0f;
    });
    if (p.states_only) {  // kept apart: the caller's state may be overwritten in place
#pragma unroll
      for (int i = 0; i < C::kState; i += 4)
        reinterpret_cast<float4*>(seg0)[(i / 4) * NT + tid] = make_float4(E[i], E[i + 1], E[i + 2], E[i + 3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < C::kState; ++i) E[i] = 0.0f;
    if (!p.states_only && active) {
      const float decay = (float)power(p.seg_tokens);
      for (int m = order == 0 ? 0 : 1; m <= order; ++m) {
        const float4* s4 = reinterpret_cast<const float4*>(seg0 + m * seg_stride);
#pragma unroll
        for (int i = 0; i < C::kState; i += 4) {
          const float4 v = s4[(i / 4) * NT + tid];
          E[i] = fmaf(E[i], decay, v.x);
          E[i + 1] = fmaf(E[i + 1], decay, v.y);
          E[i + 2] = fmaf(E[i + 2], decay, v.z);
          E[i + 3] = fmaf(E[i + 3], decay, v.w);
        }
      }
    }
  }
  // two neighbouring 16-bit values into a 128-byte-swizzled row
  auto put = [&](unsigned char* tile, int y, int piece, uint32_t v) {
    *reinterpret_cast<uint32_t*>(tile + y * 128 + ((piece ^ (y & 7)) << 4) + (lane & 3) * 4) = v;
  };
  // the state's copy, bf16, Da rows of 64-column boxes
  auto put_state = [&](int rh, int k, const float* e) {
    const int x = half * C::kCols + 8 * k;
    unsigned char* tile = sE + (x >> 6) * (DA * 128);
    const int y = erow + 16 * rh;
    put(tile, y, (x & 63) >> 3, Elem<BF>::from2(e[0], e[1]));
    put(tile, y + 8, (x & 63) >> 3, Elem<BF>::from2(e[2], e[3]));
  };
  if (!p.states_only && n_chunks > 0) {
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh)
#pragma unroll
      for (int k = 0; k < C::kCols / 8; ++k) put_state(rh, k, E + (rh * (C::kCols / 8) + k) * 4);
  }

  const uint32_t t_out = tmem + ((uint32_t)(quad * 32) << 16);  // scores, then the output
  const uint32_t t_upd = t_out + DC + half * C::kCols;
  const bool precise = r.s_out != nullptr;
  int fail = 0, it = 0;
  for (; it < n_chunks; ++it) {
    const uint32_t par = it & 1;
    const int t0 = chunk_start(it);
    const int n = min(kChunk, len - t0);
    const bool last = ends && !rev && it == n_chunks - 1;  // leave S, not beta S
    const int ex = n - (last ? 1 : 0);

    if (tid == 0) {
      fail |= !gemm::mbar_wait_poll(bar_ab, par, kWaitNs);
      if (!p.states_only) {
        gemm::tc_fence_after();
        constexpr uint32_t id = idesc<T>(kChunk, kChunk, false, false);
#pragma unroll
        for (int kk = 0; kk < DA / 16; ++kk) {
          const int off = (kk / 4) * kBoxBytes + (kk % 4) * 32;
          gemm::tc_mma(tmem, gemm::sdesc_sw128(sA + off), gemm::sdesc_sw128(sB + off), id, kk != 0);
        }
        bulk_wait_read_all();  // the last output has left sP
        gemm::tc_commit(bar_s);
      }
    }
    if (!p.states_only) {
      fail |= wait_all(bar_s, par);
      gemm::tc_fence_after();
      // decayed scores
      const int y0 = 16 * quad + (lane >> 2);
#pragma unroll
      for (int cc = 0; cc < kChunk / C::kHalves; cc += 32) {
        const int x0 = half * (kChunk / C::kHalves) + cc;
        float s[16];
        tmem_ld_rows16(t_out + x0, s);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
          for (int rr = 0; rr < 2; ++rr) {
            const int y = y0 + 8 * rr, x = x0 + 8 * k + 2 * (lane & 3);
            float w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int lag = rev ? x + e - y : y - x - e;
              const bool live = lag >= 0 && max(y, x + e) < n;
              w[e] = live ? s[4 * k + 2 * rr + e] * ptab[lag & 63] : 0.0f;
            }
            put(sP, y, (x0 >> 3) + k, Elem<T>::from2(w[0], w[1]));
          }
        }
      }
      // decayed queries, in place, as bf16 (the state's copy is)
#pragma unroll
      for (int i = 0; i < C::kABytes / 16 / NT; ++i) {
        const int piece = i * NT + tid, y = (piece >> 3) & 63;
        T* q = reinterpret_cast<T*>(sA) + piece * 8;
        float v[8];
        Elem<T>::load8(q, v);
        const float w = ptab[(rev ? n - 1 - y : y) & 63];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = y < n ? v[e] * w : 0.0f;
        Elem<BF>::store8(reinterpret_cast<BF*>(q), v);
      }
    }
    fail |= wait_all(bar_c, par);
    if (p.states_only) fail |= wait_all(bar_ab, par);
    // decayed values; part 1 is what 16 bits left out of part 0
    auto put_values = [&](int part) {
#pragma unroll
      for (int i = 0; i < C::kCBytes / 16 / NT; ++i) {
        const int piece = i * NT + tid, y = (piece >> 3) & 63;
        float v[8];
        Elem<T>::load8(reinterpret_cast<const T*>(sC) + piece * 8, v);
        const float w = y < n ? pw[rev ? y + 1 : ex - y] : 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = y < n ? v[e] * w : 0.0f;
          if (part) v[e] -= (float)T(v[e]);
        }
        Elem<T>::store8(reinterpret_cast<T*>(sW) + piece * 8, v);
      }
    };
    put_values(0);
    if (n < kChunk) {  // places past the sequence hold anything: clear them
      const uint4 z = make_uint4(0, 0, 0, 0);
      for (int i = tid; i < C::kABytes / 16; i += NT)
        if (((i >> 3) & 63) >= n) reinterpret_cast<uint4*>(sB)[i] = z;
      for (int i = tid; i < C::kCBytes / 16; i += NT)
        if (((i >> 3) & 63) >= n) reinterpret_cast<uint4*>(sC)[i] = z;
    }
    gemm::fence_async_smem();
    gemm::tc_fence_before();
    if (__syncthreads_or(fail)) break;

    constexpr uint32_t id_u = idesc<T>(DA, DC, true, true);
    if (tid == 0) {
      gemm::tc_fence_after();
      if (!p.states_only) {
        constexpr uint32_t id = idesc<BF>(kChunk, DC, false, true);
#pragma unroll
        for (int kk = 0; kk < DA / 16; ++kk)
          gemm::tc_mma(tmem, gemm::sdesc_sw128(sA + (kk / 4) * kBoxBytes + (kk % 4) * 32),
                       sdesc_mn(sE + kk * 2048, DA * 128), id, kk != 0);
      }
#pragma unroll
      for (int kk = 0; kk < kChunk / 16; ++kk)
        gemm::tc_mma(tmem + DC, sdesc_mn(sB + kk * 2048, kBoxBytes), sdesc_mn(sW + kk * 2048, kBoxBytes),
                     id_u, kk != 0);
      gemm::tc_commit(bar_u);
      if (!p.states_only) {
        constexpr uint32_t id = idesc<T>(kChunk, DC, false, true);
#pragma unroll
        for (int kk = 0; kk < kChunk / 16; ++kk)
          gemm::tc_mma(tmem, gemm::sdesc_sw128(sP + kk * 32), sdesc_mn(sC + kk * 2048, kBoxBytes), id, 1);
        gemm::tc_commit(bar_o);
      }
    }

    fail |= wait_all(bar_u, par);
    gemm::tc_fence_after();
    if (precise) {
      put_values(1);
      gemm::fence_async_smem();
      gemm::tc_fence_before();
      if (__syncthreads_or(fail)) break;
      if (tid == 0) {
        gemm::tc_fence_after();
#pragma unroll
        for (int kk = 0; kk < kChunk / 16; ++kk)
          gemm::tc_mma(tmem + DC, sdesc_mn(sB + kk * 2048, kBoxBytes), sdesc_mn(sW + kk * 2048, kBoxBytes),
                       id_u, 1);
        gemm::tc_commit(bar_l);
      }
      fail |= wait_all(bar_l, par);
      gemm::tc_fence_after();
    }
    const bool more = it + 1 < n_chunks;
    if (tid == 0 && more) load_ab(it + 1);
    const float decay = pw[ex];
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh) {
#pragma unroll
      for (int cc = 0; cc < C::kCols; cc += 32) {
        float u[16];
        tmem_ld_rows16(t_upd + ((uint32_t)(16 * rh) << 16) + cc, u);
        float* e = E + (rh * (C::kCols / 8) + cc / 8) * 4;
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = fmaf(decay, e[i], u[i]);
        if (!p.states_only && more) {
#pragma unroll
          for (int k = 0; k < 4; ++k) put_state(rh, cc / 8 + k, e + 4 * k);
        }
      }
    }
    if (p.states_only) {
      // the accumulator and the values are free once every thread is here
      gemm::tc_fence_before();
      if (__syncthreads_or(fail)) break;
      if (tid == 0 && more) load_c(it + 1);
      continue;
    }

    fail |= wait_all(bar_o, par);
    gemm::tc_fence_after();
    if (tid == 0 && more) load_c(it + 1);
    const int y0 = 16 * quad + (lane >> 2);
#pragma unroll
    for (int cc = 0; cc < C::kCols; cc += 32) {
      const int x0 = half * C::kCols + cc;
      float o[16];
      tmem_ld_rows16(t_out + x0, o);
#pragma unroll
      for (int rr = 0; rr < 2; ++rr) {
        const int y = y0 + 8 * rr;
        const bool live = y < n;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float v0 = live ? o[4 * k + 2 * rr] : 0.0f, v1 = live ? o[4 * k + 2 * rr + 1] : 0.0f;
          if (r.out_f32) {
            const int x = x0 + 8 * k + 2 * (lane & 3);
            if (t0 + y < g.T && x < r.Dc)
              *reinterpret_cast<float2*>(static_cast<float*>(r.out.data) + b * r.out.sb +
                                         (t0 + y) * r.out.st + h * r.out.sh + x) = make_float2(v0, v1);
          } else {
            put(sP + (x0 >> 6) * kBoxBytes, y, ((x0 & 63) >> 3) + k, Elem<T>::from2(v0, v1));
          }
        }
      }
    }
    gemm::fence_async_smem();
    gemm::tc_fence_before();
    if (__syncthreads_or(fail)) break;
    if (tid == 0 && !r.out_f32) {
#pragma unroll
      for (int x = 0; x < DC / 64; ++x)
        tma_store_4d(&maps.out, sP + x * kBoxBytes, 64 * x, t0, h / r.out.group, b);
      gemm::bulk_commit();
    }
  }
  if (it < n_chunks) {  // a wait gave up
    if (fail) record_status(g.status, kStatusTimeout);
    // loads in flight land before the block may exit: chunk it's, and chunk
    // it + 1's where they were started
    if (tid == 0) {
      for (int j = 0; j < 2; ++j) {
        mbar_wait_bounded(bar_ab, (it + j) & 1, gemm::kDrainWaitNs / 4);
        mbar_wait_bounded(bar_c, (it + j) & 1, gemm::kDrainWaitNs / 4);
      }
    }
  } else {
    if (p.states_only) {
      if (active && order < last_seg) {
        float4* s4 = reinterpret_cast<float4*>(seg0 + (order + 1) * seg_stride);
#pragma unroll
        for (int i = 0; i < C::kState; i += 4)
          s4[(i / 4) * NT + tid] = make_float4(E[i], E[i + 1], E[i + 2], E[i + 3]);
      }
    } else if (ends && so >= 0) {
      const float f = rev ? g.scale : 1.0f;
      each_state([&](int i, int y, int x) {
        if (y < r.Da && x < r.Dc) r.s_out[so + y * s_row + x * s_col] = f * E[i];
      });
    }
  }
  if (!p.states_only) {
    // whole chunks past the sequence's end
    const int from = t_begin + (n_tok + kChunk - 1) / kChunk * kChunk;
    const int per = r.out_f32 ? 4 : 8, pieces = r.Dc / per;
    const size_t es = r.out_f32 ? 4 : 2;
    unsigned char* o = static_cast<unsigned char*>(r.out.data) +
                       (b * r.out.sb + (h / r.out.group) * r.out.sh) * es;
    for (int i = tid; i < (t_end - from) * pieces; i += NT)
      *reinterpret_cast<uint4*>(o + ((from + i / pieces) * r.out.st + (i % pieces) * per) * es) =
          make_uint4(0, 0, 0, 0);
  }
  if (tid == 0) gemm::bulk_wait_all();
  gemm::tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    gemm::tc_fence_after();
    gemm::tmem_dealloc(tmem, C::kTmemCols);
  }
}

}  // namespace attn
}  // namespace snn
