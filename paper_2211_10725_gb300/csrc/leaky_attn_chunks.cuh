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
  static constexpr int kQBytes = kABytes > kCBytes ? kABytes : kCBytes;  // a, then values' low parts
  static constexpr int kOutBytes = kCBytes;       // >= the 8 KB of the decayed scores
  static constexpr int kTail = 1024;              // barriers, tables
  static constexpr size_t kSmem = kQBytes + kABytes + 2 * kCBytes + kEBytes + kOutBytes + kTail;
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

// 16 lanes x 32 (64) columns of TMEM: register 4k + 2r + c of lane l holds
// row l/4 + 8r, column 8k + 2(l%4) + c.  The load and its wait are one
// statement, so that nothing uses the registers before.
__device__ __forceinline__ void tmem_ld_rows(uint32_t taddr, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, "
      "%12, %13, %14, %15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]),
        "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]),
        "=f"(v[14]), "=f"(v[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_rows(uint32_t taddr, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, "
      "%12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, "
      "%30, %31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]),
        "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]),
        "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]),
        "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]),
        "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr)
      : "memory");
}
// The same places from registers; complete when the statement is.
__device__ __forceinline__ void tmem_st_rows(uint32_t taddr, const float (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, "
      "%12, %13, %14, %15, %16};\n\ttcgen05.wait::st.sync.aligned;" ::"r"(taddr),
      "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]),
      "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_rows(uint32_t taddr, const float (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, "
      "%12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, "
      "%30, %31, %32};\n\ttcgen05.wait::st.sync.aligned;" ::"r"(taddr),
      "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]),
      "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]),
      "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]), "f"(v[22]),
      "f"(v[23]), "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]),
      "f"(v[30]), "f"(v[31])
      : "memory");
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
  constexpr int NT = C::kThreads;
  constexpr bool kHalf = std::is_same<T, __half>::value;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* sA = smem;
  unsigned char* sB = sA + C::kQBytes;
  unsigned char* sC = sB + C::kABytes;
  unsigned char* sW = sC + C::kCBytes;   // decayed values
  unsigned char* sE = sW + C::kCBytes;   // the state's copy
  unsigned char* sP = sE + C::kEBytes;   // decayed scores, then the output
  uint64_t* bar = reinterpret_cast<uint64_t*>(sP + C::kOutBytes);
  uint64_t *bar_a = bar, *bar_b = bar + 1, *bar_c = bar + 2, *bar_s = bar + 3, *bar_u = bar + 4,
           *bar_o = bar + 5, *bar_x = bar + 6;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + 7);
  unsigned* top = reinterpret_cast<unsigned*>(bar + 8);  // [2] bits of the state's largest element
  float* pw = reinterpret_cast<float*>(bar + 10);  // beta^n, n = 0 .. 64
  float* lag = pw + 68;  // [128] weight of token j at token i, at i - j + 64

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int quad = warp & 3, half = warp >> 2;
  const Args& g = p.g;
  const int role = blockIdx.x % g.nroles;
  const int seg = (blockIdx.x / g.nroles) % p.nseg;
  const int row = blockIdx.x / (g.nroles * p.nseg);
  const int b = row / g.H, h = row % g.H;
  const Role& r = g.role[role];
  const RoleMaps& maps = p.map[role];
  const bool rev = r.rev != 0, out_f32 = r.out_f32 != 0, states_only = p.states_only != 0;
  const int ha = h / r.a.group, hb = h / r.b.group, hc = h / r.c.group, ho = h / r.out.group;
  const int Da = r.Da, Dc = r.Dc, T_all = g.T;
  const float scale = g.scale;

  if (tid == 0) {
    for (int i = 0; i < 7; ++i) mbar_init(&bar[i], 1);
    top[0] = top[1] = 0u;
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
  const int t_end = min(T_all, t_begin + p.seg_tokens);
  const int last_seg = len > 0 ? (len - 1) / p.seg_tokens : 0;
  const int order = rev ? last_seg - seg : seg;  // place of this segment in time
  const int n_tok = max(0, min(len, t_end) - t_begin);
  int n_chunks = (n_tok + kChunk - 1) / kChunk;
  if (states_only && order >= last_seg) n_chunks = 0;  // nothing starts after this one
  const bool active = seg <= last_seg;
  const bool ends = !states_only && r.s_out && (rev ? seg == 0 : seg == last_seg);

  auto chunk_start = [&](int it) { return t_begin + kChunk * (rev ? n_chunks - 1 - it : it); };
  auto load_a = [&](int it) {
    if (states_only) return;
    mbar_arrive_expect_tx(bar_a, C::kABytes);
#pragma unroll
    for (int x = 0; x < DA / 64; ++x)
      tma_load_4d(sA + x * kBoxBytes, &maps.a, 64 * x, chunk_start(it), ha, b, bar_a);
  };
  auto load_b = [&](int it) {
    mbar_arrive_expect_tx(bar_b, C::kABytes);
#pragma unroll
    for (int x = 0; x < DA / 64; ++x)
      tma_load_4d(sB + x * kBoxBytes, &maps.b, 64 * x, chunk_start(it), hb, b, bar_b);
  };
  auto load_c = [&](int it) {
    mbar_arrive_expect_tx(bar_c, C::kCBytes);
#pragma unroll
    for (int x = 0; x < DC / 64; ++x)
      tma_load_4d(sC + x * kBoxBytes, &maps.c, 64 * x, chunk_start(it), hc, b, bar_c);
  };
  if (tid == 0 && n_chunks > 0) {
    load_a(0);
    load_b(0);
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
  if (tid <= kChunk) pw[tid] = (float)power(tid);
  __syncthreads();
  if (tid < 128) {
    const int n = rev ? 64 - tid : tid - 64;
    lag[tid] = n >= 0 ? scale * pw[n] : 0.0f;
  }

  // this thread's part of the state: rows erow + 16*rh (+8), columns ecol + 8k (+1)
  const int erow = (C::kRowHalves == 2 ? 32 : 16) * quad + (lane >> 2);
  const int ecol = half * C::kCols + 2 * (lane & 3);
  float E[C::kRowHalves][C::kCols / 2];
  const int64_t so = (r.s_in || r.s_out) ? state_offset(g, b, h) : -1;
  const int64_t s_row = r.s_trans ? 1 : g.Dv, s_col = r.s_trans ? g.Dv : 1;
  auto each_state = [&](auto f) {  // f(value, row, column) over the thread's part
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh)
#pragma unroll
      for (int i = 0; i < C::kCols / 2; ++i)
        f(E[rh][i], erow + 16 * rh + 8 * ((i >> 1) & 1), ecol + 8 * (i >> 2) + (i & 1));
  };
  // segment states: four neighbouring registers of every thread in turn
  constexpr size_t kSegFloats = (size_t)DA * DC;
  float* const seg0 = p.seg_state + ((size_t)role * g.B * g.H + row) * p.nseg * kSegFloats;
  auto store_segment = [&](int place) {
    float4* s4 = reinterpret_cast<float4*>(seg0 + place * kSegFloats);
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh)
#pragma unroll
      for (int i = 0; i < C::kCols / 2; i += 4)
        s4[(rh * (C::kCols / 8) + i / 4) * NT + tid] =
            make_float4(E[rh][i], E[rh][i + 1], E[rh][i + 2], E[rh][i + 3]);
  };
  if (order == 0 && (p.nseg == 1 || states_only)) {
    const float f = rev ? 1.0f / scale : (len > 0 ? pw[1] : 1.0f);
    const float* s_in = so >= 0 ? r.s_in : nullptr;
    each_state([&](float& e, int y, int x) {
      e = s_in && y < Da && x < Dc ? f * s_in[so + y * s_row + x * s_col] : 0.0f;
    });
    if (states_only) store_segment(0);  // kept apart: the caller's state may be overwritten in place
  } else {
    each_state([&](float& e, int, int) { e = 0.0f; });
    if (!states_only && active) {
      const float decay = (float)power(p.seg_tokens);
      for (int m = order == 0 ? 0 : 1; m <= order; ++m) {
        const float4* s4 = reinterpret_cast<const float4*>(seg0 + m * kSegFloats);
#pragma unroll
        for (int rh = 0; rh < C::kRowHalves; ++rh)
#pragma unroll
          for (int i = 0; i < C::kCols / 2; i += 4) {
            const float4 v = s4[(rh * (C::kCols / 8) + i / 4) * NT + tid];
            E[rh][i] = fmaf(E[rh][i], decay, v.x);
            E[rh][i + 1] = fmaf(E[rh][i + 1], decay, v.y);
            E[rh][i + 2] = fmaf(E[rh][i + 2], decay, v.z);
            E[rh][i + 3] = fmaf(E[rh][i + 3], decay, v.w);
          }
      }
    }
  }

  // two neighbouring 16-bit values of this lane into row y, 16-byte piece
  // `piece`, of a tile of 128-byte swizzled rows
  auto put = [&](unsigned char* tile, int y, int piece, float v0, float v1) {
    *reinterpret_cast<uint32_t*>(tile + y * 128 + ((piece ^ (y & 7)) << 4) + (lane & 3) * 4) =
        Elem<T>::from2(v0, v1);
  };
  // The state's copy, Da rows of 64-column boxes.  fp16 has not the range of
  // a sum of products: its copy is scaled by the power of two that brings the
  // largest element to 2^10 .. 2^11, and e_back undoes it.
  float e_back = 1.0f;
  auto put_state = [&](int slot) {
    float f = 1.0f;
    if constexpr (kHalf) {
      float m = 0.0f;
      each_state([&](float& e, int, int) { m = fmaxf(m, fabsf(e)); });
      const unsigned bits = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
      if (lane == 0) atomicMax(&top[slot], bits);
      __syncthreads();
      const unsigned all = *reinterpret_cast<volatile unsigned*>(&top[slot]);
      int e = (int)(all >> 23) - 127 - 10;
      if (all == 0u || all >= 0x7f800000u) e = 0;
      e = max(e, -116);  // keeps 2^-e and 2^e normal
      f = __uint_as_float((unsigned)(127 - e) << 23);
      e_back = __uint_as_float((unsigned)(127 + e) << 23);
    }
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh) {
#pragma unroll
      for (int k = 0; k < C::kCols / 8; ++k) {
        const int x = half * C::kCols + 8 * k, y = erow + 16 * rh;
        unsigned char* tile = sE + (x >> 6) * (DA * 128);
        const float* e = &E[rh][4 * k];
        put(tile, y, (x & 63) >> 3, kHalf ? f * e[0] : e[0], kHalf ? f * e[1] : e[1]);
        put(tile, y + 8, (x & 63) >> 3, kHalf ? f * e[2] : e[2], kHalf ? f * e[3] : e[3]);
      }
    }
  };
  if (!states_only && n_chunks > 0) {
    put_state(0);
    gemm::fence_async_smem();
    __syncthreads();
  }

  const uint32_t t_acc = tmem + ((uint32_t)(quad * 32) << 16);  // scores, then the output
  const uint32_t t_upd = t_acc + DC + half * C::kCols;          // inter product, then the update
  const int y0 = 16 * quad + (lane >> 2);                       // this lane's tokens: y0, y0 + 8
  // two 16-bit parts of a bf16 value carry 16 bits of it; where the state is
  // an output, a third one makes them 24 (two of an fp16 value carry 22)
  const bool third = !kHalf && r.s_out;
  uint32_t u_phase = 0;
  int fail = 0, it = 0;
  for (; it < n_chunks; ++it) {
    const uint32_t par = it & 1;
    const int t0 = chunk_start(it);
    const int n = min(kChunk, len - t0);
    const bool last = ends && !rev && it == n_chunks - 1;  // leave S, not beta S
    const int ex = n - (last ? 1 : 0);
    const bool more = it + 1 < n_chunks;

    if (!states_only) {
      if (tid == 0) {
        if (kHalf) top[(it + 1) & 1] = 0u;
        fail |= !gemm::mbar_wait_poll(bar_a, par, kWaitNs);
        fail |= !gemm::mbar_wait_poll(bar_b, par, kWaitNs);
        gemm::tc_fence_after();
        constexpr uint32_t id_s = idesc<T>(kChunk, kChunk, false, false);
        constexpr uint32_t id_x = idesc<T>(kChunk, DC, false, true);
#pragma unroll
        for (int kk = 0; kk < DA / 16; ++kk) {
          const int off = (kk / 4) * kBoxBytes + (kk % 4) * 32;
          gemm::tc_mma(tmem, gemm::sdesc_sw128(sA + off), gemm::sdesc_sw128(sB + off), id_s, kk != 0);
        }
bulk_wait_read_all();  // the last output has left sP
        gemm::tc_commit(bar_s);
#pragma unroll
        for (int kk = 0; kk < DA / 16; ++kk)
          gemm::tc_mma(tmem + DC, gemm::sdesc_sw128(sA + (kk / 4) * kBoxBytes + (kk % 4) * 32),
                       sdesc_mn(sE + kk * 2048, DA * 128), id_x, kk != 0);
        gemm::tc_commit(bar_x);
      }
      __syncwarp();
    }
    fail |= wait_all(bar_c, par);
    if (states_only) fail |= wait_all(bar_b, par);
    // 16-bit part `PART` of the decayed values: what the parts before left of them
    auto put_values = [&](auto part, unsigned char* to) {
      constexpr int kPart = decltype(part)::value;
#pragma unroll
      for (int i = 0; i < C::kCBytes / 16 / NT; ++i) {
        const int piece = i * NT + tid, y = (piece >> 3) & 63;
        float v[8], left[8];
        Elem<T>::load8(reinterpret_cast<const T*>(sC) + piece * 8, v);
        if (n < kChunk && y >= n) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = 0.0f;
        }
        const float w = pw[max(0, rev ? y + 1 : ex - y)];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          left[e] = v[e] * w;
          if (kPart > 0) left[e] = fmaf(v[e], w, -(float)T(left[e]));
          if (kPart > 1) left[e] -= (float)T(left[e]);
        }
        Elem<T>::store8(reinterpret_cast<T*>(to) + piece * 8, left);
      }
    };
    using Part0 = std::integral_constant<int, 0>;
    using Part1 = std::integral_constant<int, 1>;
    using Part2 = std::integral_constant<int, 2>;
    put_values(Part0(), sW);
    if (!states_only) {
      fail |= wait_all(bar_s, par);
      gemm::tc_fence_after();
      // decayed scores
#pragma unroll
      for (int cc = 0; cc < kChunk / C::kHalves; cc += 32) {
        const int x0 = half * (kChunk / C::kHalves) + cc;
        float s[16];
        tmem_ld_rows(t_acc + x0, s);
        const float* w = lag + 64 + y0 - x0 - 2 * (lane & 3);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] *= w[8 * ((i >> 1) & 1) - 8 * (i >> 2) - (i & 1)];
        if (n < kChunk) {  // places past the sequence hold anything
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (max(y0 + 8 * ((i >> 1) & 1), x0 + 2 * (lane & 3) + 8 * (i >> 2) + (i & 1)) >= n) s[i] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          put(sP, y0, (x0 >> 3) + k, s[4 * k], s[4 * k + 1]);
          put(sP, y0 + 8, (x0 >> 3) + k, s[4 * k + 2], s[4 * k + 3]);
        }
      }
      fail |= wait_all(bar_x, par);
      gemm::tc_fence_after();
      // the inter product, decayed, is what the intra product adds to; the
      // scores lie in its columns, so both halves have to have read them
      if (C::kHalves == 2) asm volatile("bar.sync %0, 64;" ::"r"(1 + quad) : "memory");
      {
        float x[C::kCols / 2];
        tmem_ld_rows(t_upd, x);
        const float f0 = e_back * lag[64 + (rev ? y0 + 1 - n : y0)];
        const float f1 = e_back * lag[64 + (rev ? y0 + 9 - n : y0 + 8)];
#pragma unroll
        for (int i = 0; i < C::kCols / 2; ++i) x[i] *= (i & 2) ? f1 : f0;
        tmem_st_rows(t_acc + half * C::kCols, x);
      }
    }
    put_values(Part1(), sA);  // the scores and the inter product have read a
    if (n < kChunk) {  // clear the places past the sequence
      const uint4 z = make_uint4(0, 0, 0, 0);
      for (int i = tid; i < C::kABytes / 16; i += NT)
        if (((i >> 3) & 63) >= n) reinterpret_cast<uint4*>(sB)[i] = z;
      for (int i = tid; i < C::kCBytes / 16; i += NT)
        if (((i >> 3) & 63) >= n) reinterpret_cast<uint4*>(sC)[i] = z;
    }
    gemm::fence_async_smem();
    gemm::tc_fence_before();
    if (__syncthreads_or(fail)) break;

    auto update = [&](const unsigned char* values, uint32_t accumulate) {
      constexpr uint32_t id = idesc<T>(DA, DC, true, true);
#pragma unroll
      for (int kk = 0; kk < kChunk / 16; ++kk)
        gemm::tc_mma(tmem + DC, sdesc_mn(sB + kk * 2048, kBoxBytes),
                     sdesc_mn(values + kk * 2048, kBoxBytes), id, accumulate | (kk != 0));
    };
    if (tid == 0) {
      gemm::tc_fence_after();
      update(sW, 0);
      update(sA, 1);
      gemm::tc_commit(bar_u);
      if (!states_only) {
        constexpr uint32_t id = idesc<T>(kChunk, DC, false, true);
#pragma unroll
        for (int kk = 0; kk < kChunk / 16; ++kk)
          gemm::tc_mma(tmem, gemm::sdesc_sw128(sP + kk * 32), sdesc_mn(sC + kk * 2048, kBoxBytes), id, 1);
        gemm::tc_commit(bar_o);
      }
    }
    __syncwarp();
    fail |= wait_all(bar_u, u_phase);
    u_phase ^= 1;
    if (third) {
      put_values(Part2(), sW);
      gemm::fence_async_smem();
      if (__syncthreads_or(fail)) break;
      if (tid == 0) {
        update(sW, 1);
        gemm::tc_commit(bar_u);
      }
      __syncwarp();
      fail |= wait_all(bar_u, u_phase);
      u_phase ^= 1;
    }
    gemm::tc_fence_after();
    if (tid == 32 && more) load_a(it + 1);
    if (tid == 64 && more) load_b(it + 1);
    __syncwarp();
    const float decay = pw[ex];
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh) {
      float u[C::kCols / 2];
      tmem_ld_rows(t_upd + ((uint32_t)(16 * rh) << 16), u);
#pragma unroll
      for (int i = 0; i < C::kCols / 2; ++i) E[rh][i] = fmaf(decay, E[rh][i], u[i]);
    }
    if (states_only) {
      // the accumulator and the values are free once every thread is here
      gemm::tc_fence_before();
      if (__syncthreads_or(fail)) break;
      if (tid == 96 && more) load_c(it + 1);
      continue;
    }
    if (more) put_state((it + 1) & 1);

    fail |= wait_all(bar_o, par);
    gemm::tc_fence_after();
    if (tid == 96 && more) load_c(it + 1);
    __syncwarp();
    {
      float o[C::kCols / 2];
      tmem_ld_rows(t_acc + half * C::kCols, o);
      if (n < kChunk) {
#pragma unroll
        for (int i = 0; i < C::kCols / 2; ++i)
          if (y0 + 8 * ((i >> 1) & 1) >= n) o[i] = 0.0f;
      }
      if (out_f32) {
        float* d = static_cast<float*>(r.out.data) + b * r.out.sb + (int64_t)(t0 + y0) * r.out.st + h * r.out.sh;
#pragma unroll
        for (int i = 0; i < C::kCols / 2; i += 2) {
          const int y = 8 * ((i >> 1) & 1), x = ecol + 8 * (i >> 2);
          if (t0 + y0 + y < T_all && x < Dc)
            *reinterpret_cast<float2*>(d + y * r.out.st + x) = make_float2(o[i], o[i + 1]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < C::kCols / 8; ++k) {
          const int x = half * C::kCols + 8 * k;
          unsigned char* tile = sP + (x >> 6) * kBoxBytes;
          put(tile, y0, (x & 63) >> 3, o[4 * k], o[4 * k + 1]);
          put(tile, y0 + 8, (x & 63) >> 3, o[4 * k + 2], o[4 * k + 3]);
        }
      }
    }
    gemm::fence_async_smem();
    gemm::tc_fence_before();
    if (__syncthreads_or(fail)) break;
    if (tid == 0 && !out_f32) {
#pragma unroll
      for (int x = 0; x < DC / 64; ++x)
        tma_store_4d(&maps.out, sP + x * kBoxBytes, 64 * x, t0, ho, b);
      gemm::bulk_commit();
    }
  }
  if (it < n_chunks) {  // a wait gave up
    if (fail) record_status(g.status, kStatusTimeout);
    // loads in flight land before the block may exit: chunk it's, and chunk
    // it + 1's where they were started
    if (tid == 0) {
      for (int j = 0; j < 2; ++j) {
        if (!states_only) mbar_wait_bounded(bar_a, (it + j) & 1, gemm::kDrainWaitNs / 4);
        mbar_wait_bounded(bar_b, (it + j) & 1, gemm::kDrainWaitNs / 4);
        mbar_wait_bounded(bar_c, (it + j) & 1, gemm::kDrainWaitNs / 4);
      }
    }
  } else if (states_only) {
    if (active && order < last_seg) store_segment(order + 1);
  } else if (ends && so >= 0) {
    const float f = rev ? scale : 1.0f;
    float* s_out = r.s_out + so;
    each_state([&](float& e, int y, int x) {
      if (y < Da && x < Dc) s_out[y * s_row + x * s_col] = f * e;
    });
  }
  if (!states_only) {
    // whole chunks past the sequence's end
    const int from = t_begin + (n_tok + kChunk - 1) / kChunk * kChunk;
    const int per = out_f32 ? 4 : 8, pieces = Dc / per;
    const size_t es = out_f32 ? 4 : 2;
    unsigned char* o = static_cast<unsigned char*>(r.out.data) + (b * r.out.sb + ho * r.out.sh) * es;
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
