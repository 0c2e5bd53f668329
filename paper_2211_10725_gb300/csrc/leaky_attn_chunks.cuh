// Leaky attention in chunks on the tensor cores.
//
// With E the state a chunk starts from, already decayed to its first token,
// the recurrence over n <= 64 tokens is four products (i, j count tokens in
// the direction of time of the role, see leaky_attn.cuh):
//   scores  s_ij = a_i . b_j                                          [64 x 64]
//   inter   X = (scale beta^i) E^T a_i                                [Dc x 64]
//   intra   O = X + sum_{j <= i} (scale beta^(i-j) s_ij) c_j          [Dc x 64]
//   update  E^T <- beta^n E^T + sum_j (beta^(n-j) c_j) b_j^T          [Dc x Da]
// A block walks the chunks of one head in order with E in fp32 registers, so
// every token is read once and the state never leaves the SM.  The last three
// products are taken transposed, with the Dc channels as the rows: a 128-wide
// head then fills the tensor core's 128 rows although a chunk has 64 tokens,
// and the state's 16-bit parts are an operand in tensor memory (in shared
// memory for a 64-wide head).  Operands land by TMA as 64-token, 64-element
// boxes (128-byte swizzle); the same box of b is the K-major operand of the
// scores and the MN-major one of the update.  Per chunk one thread issues the
// MMAs in two groups, with the block's work between: the decayed scores and
// values go back to shared memory as 16-bit operands, the inter product is
// decayed in place; then the output leaves by TMA and the state is updated.
// Two blocks (128-wide heads) or three (64-wide) share an SM and fill each
// other's waits; 64-token chunks are what lets two working sets fit.
//
// The output is rounded to 16 bits.  The decayed scores and the state are two
// 16-bit parts each in their products, multiplied in turn: rounded to one, each
// would add as much error as the output's own rounding (2-norm, bf16: 0.0023
// instead of 0.0017; an output of few tokens shows a single score's in full).
// The decayed values are two 16-bit parts each (v w = hi + lo with products
// and residuals exact in packed 16-bit arithmetic), multiplied in turn, so a
// state keeps 16 bits or more of each term; where a bf16 state is an output, a
// third part makes them 24 (fp16: two make 22).  fp16 has not the range of a sum
// of products: its values, scores and state are scaled by a power of two each
// chunk.
//
// Few heads and many tokens: the tokens are cut into segments, a first kernel
// (attn_segments: update products only) finds each segment's own contribution
// to the state; a second (attn_segment_scan), where there are more than a few,
// the state each one starts from.
//
// What bounds it, measured (128 x 128): with two blocks on every SM issue slots and
// the tensor core's operand reads are each busy half of the time, and the rest is
// the chain of a chunk's products and barriers.  8 x 4096 tokens of 38 heads, which
// are two blocks for each of 152 SMs: bf16 239 us, the tensors' bytes at 5.3 TB/s,
// 0.79 of the measured copy rate (201 with one part each of the scores and the
// state, 219 with two of the scores alone); fp16 314 (its three scalings a chunk
// cost a barrier each).  2 x 4096 tokens of 32 heads, bf16: 97.  A block alone on its
// SM takes 2.6 us a chunk, one of two 3.7.
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
  int scanned;          // attn_segment_scan has run
  float* seg_state;     // [role][B*H][nseg] states in fragment order
};

template <int DA, int DC>
struct Cfg {
  static constexpr int kThreads = (DA == 128 || DC == 128) ? 256 : 128;
  static constexpr int kHalves = kThreads / 128;   // column halves of an accumulator
  static constexpr int kRowHalves = DC / 64;       // 16-lane halves of a warp's channels
  static constexpr int kCols = DA / kHalves;       // state columns of a warp: neighbours,
  // or, of 128 in two halves, 32 in each 64, so that every warp has read the
  // upper 64 columns of its update where it puts the state's second parts
  static constexpr bool kSplit = DA == 128 && kHalves == 2;
  static constexpr int kStep = kSplit ? 32 : kCols;  // from one half's first column to the other's
  static constexpr int kToks = kChunk / kHalves;   // tokens (score columns) of a warp
  static constexpr int kABytes = kChunk * DA * 2;
  static constexpr int kCBytes = kChunk * DC * 2;
  static constexpr bool kStateTmem = DC == 128;    // where the state's 16-bit parts are
  static constexpr int kEBytes = kStateTmem ? 0 : 2 * DA * DC * 2;
  static constexpr int kOutBytes = kCBytes;        // decayed scores (8 KB a part), then the output
  static constexpr int kTail = 1024;               // barriers, tables
  // b has two stages, as its last use in a chunk is the latest
  static constexpr int kBStages = 2;
  // a's place, big enough to take a third part of the values after a's last use
  static constexpr int kQBytes = kABytes > kCBytes ? kABytes : kCBytes;
  static constexpr size_t kSmem = kQBytes + kBStages * kABytes + 3 * kCBytes + kEBytes + kOutBytes + kTail;
  // attn_segments: two stages of b and c, the parts of the decayed values
  static constexpr size_t kSegSmem = 2 * (kABytes + kCBytes) + 2 * kCBytes + kTail;
  static constexpr uint32_t kSegTmemCols = 2 * DA;
  // tensor memory: output, update (scores in its first 64 columns), first
  // parts of the state; the second ones behind, or in the update's upper half
  static constexpr uint32_t kTmemCols = kStateTmem ? 256 : (DA == 64 ? 128 : 256);
  static constexpr int kBlocksPerSm = kThreads == 128 ? 3 : 2;
  static constexpr int kSegBlocksPerSm = kThreads == 128 ? 4 : 2;
};

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z,
                                            int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
          smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
      : "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}

__device__ __forceinline__ void tma_store_4d(const CUtensorMap* map, const void* src, int x, int y,
                                             int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(
          reinterpret_cast<uint64_t>(map)),
      "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}

// Bring a box into L2, ahead of the load that will want it.
__device__ __forceinline__ void tma_prefetch_4d(const CUtensorMap* map, int x, int y, int z, int w) {
  asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global.tile [%0, {%1, %2, %3, %4}];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(x), "r"(y), "r"(z), "r"(w)
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

// 16 lanes x 4*N/2 32-bit columns from registers: register 2k + r of lane l
// goes to row l/4 + 8r, column 4k + l%4 (pairs of 16-bit values of an operand).
__device__ __forceinline__ void tmem_st_pairs(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
      : "memory");
}
__device__ __forceinline__ void tmem_st_pairs(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, "
      "%12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
      "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// Four 8x8 blocks of 16-bit values, transposed into shared memory: lane l
// gives the address of row l%8 of block l/8.
__device__ __forceinline__ void stmatrix_t(void* row, uint32_t r0, uint32_t r1, uint32_t r2,
                                           uint32_t r3) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(
                   smem_u32(row)),
               "r"(r0), "r"(r1), "r"(r2), "r"(r3)
               : "memory");
}

// One lane of a whole warp.
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t e;
  asm volatile(
      "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(e));
  return e;
}

// MMAs and commits of the elected lane, written for the whole warp: the
// operands stay uniform across it, which the instruction wants (a lane of its
// own would move each descriptor between register files, about 75 cycles an
// MMA).  D (tensor memory) [+]= A * B with A and B in shared memory (ss) or A in
// tensor memory, K-major (ts).
__device__ __forceinline__ void mma_ss(uint32_t e, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(e)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t e, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(e)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t e, uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(
          smem_u32(bar)),
      "r"(e)
      : "memory");
}

// v w = hi + lo in packed 16-bit arithmetic, for a weight in two parts: the
// residual of hi is exact (a product of two significands is twice as wide).
__device__ __forceinline__ void split_product(__nv_bfloat162 v, __nv_bfloat162 w1, __nv_bfloat162 w2,
                                              __nv_bfloat162& hi, __nv_bfloat162& lo) {
  hi = __hmul2_rn(v, w1);
  lo = __hfma2(v, w2, __hfma2(v, w1, __hneg2(hi)));
}
__device__ __forceinline__ void split_product(__half2 v, __half2 w1, __half2 w2, __half2& hi, __half2& lo) {
  hi = __hmul2_rn(v, w1);
  lo = __hfma2(v, w2, __hfma2(v, w1, __hneg2(hi)));
}

// x and y as two 16-bit parts each.
__device__ __forceinline__ float2 minus2(float x, float y, float a, float b) {
  uint64_t w, v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(w) : "f"(x), "f"(y));
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(-a), "f"(-b));
  asm("add.rn.f32x2 %0, %0, %1;" : "+l"(w) : "l"(v));
  float2 d;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(w));
  return d;
}
template <typename T>
__device__ __forceinline__ uint32_t two_parts(float x, float y, uint32_t& rest) {
  const uint32_t first = Elem<T>::from2(x, y);
  float2 d;
  if constexpr (std::is_same<T, __half>::value) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&first));
    d = minus2(x, y, f.x, f.y);
  } else {
    d = minus2(x, y, __uint_as_float(first << 16), __uint_as_float(first & 0xffff0000u));
  }
  rest = Elem<T>::from2(d.x, d.y);
  return first;
}

template <typename T>
struct Pair;
template <>
struct Pair<__nv_bfloat16> {
  using type = __nv_bfloat162;
};
template <>
struct Pair<__half> {
  using type = __half2;
};

// x^n for 0 <= x <= 1, n >= 0.  The error is n |log2 x| 2^-24, i.e. |log2 of the
// result| units: a weight that counts is as good as an fp32 product.
__device__ __forceinline__ float power(float x, int n) { return n == 0 ? 1.0f : exp2f((float)n * log2f(x)); }

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

// beta^n by direction: at 64 + n (64 - n for a role backwards in time), n = 0 ..
// 64, zeros on the other side; and in two 16-bit parts.
template <typename T>
struct Decays {
  float lag[2 * kChunk + 1];
  typename Pair<T>::type parts[kChunk + 1];

  __device__ __forceinline__ void fill(float beta, bool rev, int tid) {
    if (tid > kChunk) return;
    const float w = power(beta, tid);
    const T hi = T(w);
    parts[tid] = typename Pair<T>::type(hi, T(w - (float)hi));
    if (tid > 0) lag[rev ? kChunk + tid : kChunk - tid] = 0.0f;
    lag[rev ? kChunk - tid : kChunk + tid] = w;
  }
  __device__ __forceinline__ float of(int n, bool rev) const { return lag[rev ? kChunk - n : kChunk + n]; }
};

// Where a block is: which role, head and segment, and that segment's tokens.
struct Place {
  int role, seg, row, b, h;
  int len;        // tokens of the sequence
  int begin;      // first token of the segment
  int tokens;     // tokens of it that exist
  int chunks;
  int last_seg;   // segment of the sequence's last token
  int order;      // place of this segment in time, 0 .. last_seg

  __device__ __forceinline__ explicit Place(const ChunkArgs& p) {
    role = blockIdx.x % p.g.nroles;
    seg = (blockIdx.x / p.g.nroles) % p.nseg;
    row = blockIdx.x / (p.g.nroles * p.nseg);
    b = row / p.g.H;
    h = row % p.g.H;
  }
  __device__ __forceinline__ void measure(const ChunkArgs& p, bool rev) {
    len = seq_len(p.g, b);
    begin = seg * p.seg_tokens;
    tokens = max(0, min(len, min(p.g.T, begin + p.seg_tokens)) - begin);
    chunks = (tokens + kChunk - 1) / kChunk;
    last_seg = len > 0 ? (len - 1) / p.seg_tokens : 0;
    order = rev ? last_seg - seg : seg;
  }
  __device__ __forceinline__ int start(int it, bool rev) const {  // first token of chunk it in time
    return begin + kChunk * (rev ? chunks - 1 - it : it);
  }
};

// A thread's part of a head's transposed state: channels row + 16*rh (+8) of c,
// columns col + 8k (+1) of a and b (split columns: from k = 4 on 32 further).
template <int DA, int DC>
struct State {
  using C = Cfg<DA, DC>;
  float e[C::kRowHalves][C::kCols / 2];
  int row, col;

  __device__ __forceinline__ State(int quad, int half, int lane)
      : row((C::kRowHalves == 2 ? 32 : 16) * quad + (lane >> 2)), col(half * C::kStep + 2 * (lane & 3)) {
    each([](float& x, int, int) { x = 0.0f; });
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) {  // f(value, channel, column)
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh)
#pragma unroll
      for (int i = 0; i < C::kCols / 2; ++i)
        f(e[rh][i], row + 16 * rh + 8 * ((i >> 1) & 1),
          col + 8 * (i >> 2) + (C::kSplit && i >= 16 ? 32 : 0) + (i & 1));
  }
  // e = f * the caller's state (zeros where there is none)
  __device__ __forceinline__ void load(const Args& g, const Role& r, int b, int h, float f) {
    const int64_t so = r.s_in ? state_offset(g, b, h) : -1;
    if (so < 0) return;
    const float* s = r.s_in + so;
    const int64_t sr = r.s_trans ? g.Dv : 1, sc = r.s_trans ? 1 : g.Dv;
    each([&](float& x, int y, int c) {
      if (y < r.Dc && c < r.Da) x = f * s[y * sr + c * sc];
    });
  }
  __device__ __forceinline__ void store(const Args& g, const Role& r, int b, int h, float f) {
    const int64_t so = state_offset(g, b, h);
    if (so < 0) return;
    float* s = r.s_out + so;
    const int64_t sr = r.s_trans ? g.Dv : 1, sc = r.s_trans ? 1 : g.Dv;
    each([&](float& x, int y, int c) {
      if (y < r.Dc && c < r.Da) s[y * sr + c * sc] = f * x;
    });
  }
  // segment states: four neighbouring registers of every thread in turn
  __device__ __forceinline__ void put_segment(float* at, int tid) {
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh)
#pragma unroll
      for (int i = 0; i < C::kCols / 2; i += 4)
        reinterpret_cast<float4*>(at)[(rh * (C::kCols / 8) + i / 4) * C::kThreads + tid] =
            make_float4(e[rh][i], e[rh][i + 1], e[rh][i + 2], e[rh][i + 3]);
  }
  __device__ __forceinline__ void add_segment(const float* at, int tid, float decay) {  // e = decay e + it
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh)
#pragma unroll
      for (int i = 0; i < C::kCols / 2; i += 4) {
        const float4 v =
            reinterpret_cast<const float4*>(at)[(rh * (C::kCols / 8) + i / 4) * C::kThreads + tid];
        e[rh][i] = fmaf(e[rh][i], decay, v.x);
        e[rh][i + 1] = fmaf(e[rh][i + 1], decay, v.y);
        e[rh][i + 2] = fmaf(e[rh][i + 2], decay, v.z);
        e[rh][i + 3] = fmaf(e[rh][i + 3], decay, v.w);
      }
  }
  // e = decay e + f * the update product in tensor memory (at: the thread's half)
  __device__ __forceinline__ void add_update(uint32_t at, float decay, float f) {
    constexpr int kRun = C::kSplit ? 16 : C::kCols / 2;  // registers of neighbouring columns
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh)
#pragma unroll
      for (int j = 0; j < C::kCols / 2; j += kRun) {
        float u[kRun];
        tmem_ld_rows(at + ((uint32_t)(16 * rh) << 16) + (j ? 64 : 0), u);
#pragma unroll
        for (int i = 0; i < kRun; ++i) e[rh][j + i] = fmaf(decay, e[rh][j + i], f * u[i]);
      }
  }
};

// The decayed values of a chunk, hi and lo parts: a piece of 8 with its weight
// in two parts (a place past the sequence counts as zeros), scaled up by f.
template <typename T>
__device__ __forceinline__ void split_piece(const unsigned char* values, int piece, bool live,
                                            typename Pair<T>::type w, float f, uint4& hi, uint4& lo) {
  using T2 = typename Pair<T>::type;
  uint4 v = reinterpret_cast<const uint4*>(values)[piece];
  if (!live) v = make_uint4(0, 0, 0, 0);
  if constexpr (std::is_same<T, __half>::value) {
    const __half2 up = __float2half2_rn(f);
    __half2* p = reinterpret_cast<__half2*>(&v);
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = __hmul2(p[e], up);
  }
  const T2 w1 = T2(w.x, w.x), w2 = T2(w.y, w.y);
  const T2* vp = reinterpret_cast<const T2*>(&v);
  T2 *hp = reinterpret_cast<T2*>(&hi), *lp = reinterpret_cast<T2*>(&lo);
#pragma unroll
  for (int e = 0; e < 4; ++e) split_product(vp[e], w1, w2, hp[e], lp[e]);
}
// What the two parts left of v w, to 16 bits.
template <typename T>
__device__ __forceinline__ uint4 third_part(const unsigned char* values, int piece, bool live, float w,
                                            uint4 hi, uint4 lo) {
  float v[8], a[8], b[8];
  Elem<T>::load8(reinterpret_cast<const T*>(values) + piece * 8, v);
  Elem<T>::load8(reinterpret_cast<const T*>(&hi), a);
  Elem<T>::load8(reinterpret_cast<const T*>(&lo), b);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = live ? fmaf(v[e], w, -a[e]) - b[e] : 0.0f;
  uint4 out;
  Elem<T>::store8(reinterpret_cast<T*>(&out), v);
  return out;
}

__device__ __forceinline__ float power_of_2(int e) { return __uint_as_float((unsigned)(127 + e) << 23); }

// e for which the block's largest m lies in 2^(e+to) .. 2^(e+to+1) (0 where it is
// zero or not finite).  Every thread of the block calls; *slot is 0 before.
__device__ __forceinline__ int exponent_of_all(unsigned* slot, float m, int lane, int to) {
  const unsigned bits = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
  if (lane == 0) atomicMax(slot, bits);
  __syncthreads();
  const unsigned all = *reinterpret_cast<volatile unsigned*>(slot);
  return all == 0u || all >= 0x7f800000u ? 0 : (int)(all >> 23) - 127 - to;
}

// fp16 keeps parts of a decayed value to 2^-25.  e for which 2^-e brings a
// chunk's largest value to 2^14 .. 2^15 (no further up than 2^15, fp16's largest
// power), so that they go by that value; the update product is 2^-e too large.
template <int PIECES>
__device__ __forceinline__ int values_exponent(unsigned* slot, const unsigned char* values, int n, int tid,
                                               int threads) {
  __half2 m = __float2half2_rn(0.0f);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int piece = i * threads + tid;
    uint4 v = reinterpret_cast<const uint4*>(values)[piece];
    if (((piece >> 3) & 63) >= n) v = make_uint4(0, 0, 0, 0);
    const __half2* p = reinterpret_cast<const __half2*>(&v);
#pragma unroll
    for (int e = 0; e < 4; ++e) m = __hmax2(m, __habs2(p[e]));
  }
  const float most = fmaxf(__low2float(m), __high2float(m));
  return min(max(exponent_of_all(slot, most, tid & 31, 14), -15), 0);
}

// Zero the places past the sequence's end in a tile of 128-byte rows.
__device__ __forceinline__ void clear_rows(unsigned char* tile, int bytes, int n, int tid, int threads) {
  for (int i = tid; i < bytes / 16; i += threads)
    if (((i >> 3) & 63) >= n) reinterpret_cast<uint4*>(tile)[i] = make_uint4(0, 0, 0, 0);
}

// The first kernel of a segmented run: each segment's state after its own
// tokens (the first one's from the caller's state, kept too, because that may
// be overwritten in place).  The tiles of b and c have two stages, and the
// state is updated from one accumulator while the next chunk's products fill
// the other.  2 x 4096 tokens of 32 heads in four segments take 31 us, 3.2 TB/s: two
// blocks of an SM take 1.9 us a chunk each, bound by the chain from the split of
// the values through their products.  One block on an SM with the split
// pipelined as well (twice the shared memory) took 1.1.
template <typename T, int DA, int DC>
__global__ void __launch_bounds__(Cfg<DA, DC>::kThreads, Cfg<DA, DC>::kSegBlocksPerSm)
    attn_segments(const __grid_constant__ ChunkArgs p) {
  using C = Cfg<DA, DC>;
  constexpr int NT = C::kThreads;
  constexpr bool kHalf = std::is_same<T, __half>::value;
  constexpr int kStage = C::kABytes + C::kCBytes;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* sW = smem + 2 * kStage;
  unsigned char* sL = sW + C::kCBytes;
  uint64_t* bar = reinterpret_cast<uint64_t*>(sL + C::kCBytes);  // [2] loads, [1] update
  uint64_t* bar_u = bar + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + 3);
  unsigned* top = reinterpret_cast<unsigned*>(bar + 4);  // [2] bits of the largest value (fp16)
  Decays<T>& decays = *reinterpret_cast<Decays<T>*>(bar + 5);
  unsigned char* sT = sL + C::kCBytes + C::kTail;  // third parts, where there are any

  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int quad = warp & 3, half = warp >> 2;
  const Args& g = p.g;
  Place at(p);
  const Role& r = g.role[at.role];
  const RoleMaps& maps = p.map[at.role];
  const bool rev = r.rev != 0;
  const int hb = at.h / r.b.group, hc = at.h / r.c.group;

  if (tid == 32 && g.T > 0) {
    prefetch_map(&maps.b);
    prefetch_map(&maps.c);
  }
  if (tid == 0) {
    for (int i = 0; i < 3; ++i) mbar_init(&bar[i], 1);
    top[0] = top[1] = 0u;
    fence_barrier_init();
  }
  __syncwarp();
  if (warp == 0) gemm::tmem_alloc(tmem_slot, C::kSegTmemCols);
  gemm::tc_fence_before();
  __syncthreads();
  gemm::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_dep_wait();

  const float beta = g.beta[at.h];
  at.measure(p, rev);
  const bool wanted = at.seg <= at.last_seg && at.order < at.last_seg;  // something starts after it
  const int n_chunks = wanted ? at.chunks : 0;
  auto load = [&](int it) {
    unsigned char* stage = smem + (it & 1) * kStage;
    const int t0 = at.start(it, rev);
    mbar_arrive_expect_tx(&bar[it & 1], kStage);
#pragma unroll
    for (int x = 0; x < DA / 64; ++x)
      tma_load_4d(stage + x * kBoxBytes, &maps.b, 64 * x, t0, hb, at.b, &bar[it & 1]);
#pragma unroll
    for (int x = 0; x < DC / 64; ++x)
      tma_load_4d(stage + C::kABytes + x * kBoxBytes, &maps.c, 64 * x, t0, hc, at.b, &bar[it & 1]);
  };
  if (tid == 0) {
    if (n_chunks > 0) load(0);
    if (n_chunks > 1) load(1);
  }
  decays.fill(beta, rev, tid);
  State<DA, DC> state(quad, half, lane);
  float* const seg0 = p.seg_state + ((size_t)at.role * g.B * g.H + at.row) * p.nseg * (size_t)(DA * DC);
  if (at.order == 0) {
    state.load(g, r, at.b, at.h, rev ? 1.0f / g.scale : (at.len > 0 ? beta : 1.0f));
    state.put_segment(seg0, tid);
  }
  __syncthreads();

  const uint32_t t_upd = tmem + ((uint32_t)(quad * 32) << 16) + half * C::kStep;
  const bool third = !kHalf && r.s_out;
  float back_last = 1.0f;
  int fail = 0, it = 0, n_last = 0;
  for (; it < n_chunks; ++it) {
    const int n = min(kChunk, at.len - at.start(it, rev));
    unsigned char* sB = smem + (it & 1) * kStage;
    unsigned char* sC = sB + C::kABytes;
    if (it > 0) {  // the last products have read their operands
      fail |= wait_all(bar_u, (it - 1) & 1);
      if (tid == 32 && it + 1 < n_chunks) load(it + 1);
      __syncwarp();
    }
    fail |= wait_all(&bar[it & 1], (it >> 1) & 1);
    float up = 1.0f, back = 1.0f;
    if constexpr (kHalf) {
      if (tid == 0) top[(it + 1) & 1] = 0u;
      const int e = values_exponent<C::kCBytes / 16 / NT>(&top[it & 1], sC, n, tid, NT);
      up = power_of_2(-e);
      back = power_of_2(e);
    }
#pragma unroll
    for (int i = 0; i < C::kCBytes / 16 / NT; ++i) {
      const int piece = i * NT + tid, y = (piece >> 3) & 63;
      const int lag = max(0, rev ? y + 1 : n - y);
      uint4 hi, lo;
      split_piece<T>(sC, piece, y < n, decays.parts[lag], up, hi, lo);
      reinterpret_cast<uint4*>(sW)[piece] = hi;
      reinterpret_cast<uint4*>(sL)[piece] = lo;
      if (third)
        reinterpret_cast<uint4*>(sT)[piece] = third_part<T>(sC, piece, y < n, decays.of(lag, rev), hi, lo);
    }
    if (n < kChunk) clear_rows(sB, C::kABytes, n, tid, NT);
    gemm::fence_async_smem();
    gemm::tc_fence_before();
    if (__syncthreads_or(fail)) break;
    if (warp == 0) {
      gemm::tc_fence_after();
      const uint32_t e = elect_one();
      constexpr uint32_t id = idesc<T>(DC, DA, true, true);
#pragma unroll
      for (int part = 0; part < 3; ++part) {
        if (part == 2 && !third) continue;
        const unsigned char* values = part == 0 ? sW : part == 1 ? sL : sT;
#pragma unroll
        for (int kk = 0; kk < kChunk / 16; ++kk)
          mma_ss(e, tmem + (it & 1) * DA, sdesc_mn(values + kk * 2048, kBoxBytes),
                 sdesc_mn(sB + kk * 2048, kBoxBytes), id, part | kk);
      }
      mma_commit(e, bar_u);
    }
    if (it > 0) {
      gemm::tc_fence_after();
      state.add_update(t_upd + ((it - 1) & 1) * DA, decays.of(n_last, rev), back_last);
    }
    n_last = n;
    back_last = back;
  }
  if (it < n_chunks) {  // a wait gave up: loads in flight land before the block may exit
    if (fail) record_status(g.status, kStatusTimeout);
    if (tid == 0)
      for (int j = it; j < min(it + 2, n_chunks); ++j)
        mbar_wait_bounded(&bar[j & 1], (j >> 1) & 1, gemm::kDrainWaitNs);
  } else if (wanted) {
    if (n_chunks > 0) {
      if (wait_all(bar_u, (n_chunks - 1) & 1)) record_status(g.status, kStatusTimeout);
      gemm::tc_fence_after();
      state.add_update(t_upd + ((n_chunks - 1) & 1) * DA, decays.of(n_last, rev), back_last);
    }
    state.put_segment(seg0 + (size_t)(at.order + 1) * (DA * DC), tid);
  }
  gemm::tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    gemm::tc_fence_after();
    gemm::tmem_dealloc(tmem, C::kSegTmemCols);
  }
}

// The second kernel of a segmented run: in place, the state that the segment at
// each place in time starts from.  At 0 is the first one's; from 1 on, what the
// segment before it added (1: with the first one's start), so
//   E_1 = s_1,  E_m = beta^tokens E_{m-1} + s_m.
// Every thread takes four neighbouring floats through all places, eight loads
// in flight (19 places of 16 heads: 19 MB read from a cold cache in 8 us).
constexpr int kScanThreads = 256;
__global__ void __launch_bounds__(kScanThreads) attn_segment_scan(const __grid_constant__ ChunkArgs p,
                                                                  int floats) {
  grid_dep_wait();
  const int per = floats / (4 * kScanThreads);  // blocks of a head
  const int head = blockIdx.x / per;            // role * B * H + row
  const int row = head % (p.g.B * p.g.H);
  const int len = seq_len(p.g, row / p.g.H);
  const int last_seg = len > 0 ? (len - 1) / p.seg_tokens : 0;
  if (last_seg < 2) return;
  const float decay = power(p.g.beta[row % p.g.H], p.seg_tokens);
  const size_t step = (size_t)floats / 4;
  float4* s = reinterpret_cast<float4*>(p.seg_state + (size_t)head * p.nseg * floats) +
              (blockIdx.x % per) * kScanThreads + threadIdx.x;
  float4 e = s[step];
  for (int m = 2; m <= last_seg; m += 8) {
    float4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (m + i <= last_seg) v[i] = s[(m + i) * step];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (m + i > last_seg) break;
      e.x = fmaf(e.x, decay, v[i].x);
      e.y = fmaf(e.y, decay, v[i].y);
      e.z = fmaf(e.z, decay, v[i].z);
      e.w = fmaf(e.w, decay, v[i].w);
      s[(m + i) * step] = e;
    }
  }
}

template <typename T, int DA, int DC>
__global__ void __launch_bounds__(Cfg<DA, DC>::kThreads, Cfg<DA, DC>::kBlocksPerSm)
    attn_chunks(const __grid_constant__ ChunkArgs p) {
  using C = Cfg<DA, DC>;
  constexpr int NT = C::kThreads;
  constexpr int kStorer = NT - 32;  // thread that issues and awaits the output's copies
  constexpr bool kHalf = std::is_same<T, __half>::value;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* sA = smem;
  unsigned char* sB2 = sA + C::kQBytes;                   // the stages of b
  unsigned char* sC = sB2 + C::kBStages * C::kABytes;
  unsigned char* sW = sC + C::kCBytes;                    // decayed values, high parts
  unsigned char* sL = sW + C::kCBytes;                    // low parts
  unsigned char* sP = sL + C::kCBytes;                    // decayed scores, then the output
  unsigned char* sE = sP + C::kOutBytes;                  // the state's parts (64-wide heads)
  // second parts of the decayed scores: beside the first ones, or where the
  // state's were (the inter product has read them)
  unsigned char* sQ = C::kStateTmem ? sP + kBoxBytes : sE;
  // an fp32 output is twice as long: it goes where the decayed values were
  unsigned char* sO32 = sW;
  uint64_t* bar = reinterpret_cast<uint64_t*>(sE + C::kEBytes);
  uint64_t *bar_a = bar, *bar_b = bar + 1, *bar_c = bar + 3, *bar_s = bar + 4, *bar_u = bar + 5,
           *bar_o = bar + 6, *bar_x = bar + 7, *bar_p = bar + 8;  // bar_b: one for each stage
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + 9);
  unsigned* top = reinterpret_cast<unsigned*>(bar + 10);   // [2] bits of the state's largest element
  unsigned* peak = reinterpret_cast<unsigned*>(bar + 11);  // [2] of the scores'
  unsigned* most = reinterpret_cast<unsigned*>(bar + 12);  // [2] and of the values'
  Decays<T>& decays = *reinterpret_cast<Decays<T>*>(bar + 13);

  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int quad = warp & 3, half = warp >> 2;
  const Args& g = p.g;
  Place at(p);
  const Role& r = g.role[at.role];
  const RoleMaps& maps = p.map[at.role];
  const bool rev = r.rev != 0, out_f32 = r.out_f32 != 0;
  const int b = at.b, h = at.h;
  const int ha = h / r.a.group, hb = h / r.b.group, hc = h / r.c.group, ho = h / r.out.group;
  const int Dc = r.Dc, T_all = g.T;
  const float scale = g.scale;

  if (tid == 32 && g.T > 0) {
    prefetch_map(&maps.a);
    prefetch_map(&maps.b);
    prefetch_map(&maps.c);
  }
  if (tid == 0) {
    for (int i = 0; i < 9; ++i) mbar_init(&bar[i], 1);
    top[0] = top[1] = peak[0] = peak[1] = most[0] = most[1] = 0u;
    fence_barrier_init();
  }
  __syncwarp();
  if (warp == 0) gemm::tmem_alloc(tmem_slot, C::kTmemCols);
  gemm::tc_fence_before();
  __syncthreads();
  gemm::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_dep_wait();

  const float beta = g.beta[h];
  at.measure(p, rev);
  const int n_chunks = at.chunks;
  const bool ends = r.s_out && (rev ? at.seg == 0 : at.seg == at.last_seg);

  auto load_a = [&](int it) {
    mbar_arrive_expect_tx(bar_a, C::kABytes);
#pragma unroll
    for (int x = 0; x < DA / 64; ++x)
      tma_load_4d(sA + x * kBoxBytes, &maps.a, 64 * x, at.start(it, rev), ha, b, bar_a);
  };
  auto load_b = [&](int it) {
    const int stage = it % C::kBStages;
    unsigned char* to = sB2 + stage * C::kABytes;
    mbar_arrive_expect_tx(bar_b + stage, C::kABytes);
#pragma unroll
    for (int x = 0; x < DA / 64; ++x)
      tma_load_4d(to + x * kBoxBytes, &maps.b, 64 * x, at.start(it, rev), hb, b, bar_b + stage);
  };
  auto load_c = [&](int it) {
    mbar_arrive_expect_tx(bar_c, C::kCBytes);
#pragma unroll
    for (int x = 0; x < DC / 64; ++x)
      tma_load_4d(sC + x * kBoxBytes, &maps.c, 64 * x, at.start(it, rev), hc, b, bar_c);
  };
  // a and c of chunk it into L2: their buffers free up only shortly before
  // they are wanted, so the loads themselves should not have to go to HBM
  auto prefetch = [&](int it) {
    if (it >= n_chunks) return;
    const int t0 = at.start(it, rev);
#pragma unroll
    for (int x = 0; x < DC / 64; ++x) tma_prefetch_4d(&maps.c, 64 * x, t0, hc, b);
#pragma unroll
    for (int x = 0; x < DA / 64; ++x) tma_prefetch_4d(&maps.a, 64 * x, t0, ha, b);
  };
  if (tid == 0 && n_chunks > 0) {
    load_a(0);
    load_b(0);
    load_c(0);
    prefetch(1);
  }

  decays.fill(beta, rev, tid);
  __syncthreads();
  State<DA, DC> state(quad, half, lane);
  const float* const seg0 =
      p.seg_state + ((size_t)at.role * g.B * g.H + at.row) * p.nseg * (size_t)(DA * DC);
  if (p.nseg == 1) {
    state.load(g, r, b, h, rev ? 1.0f / scale : (at.len > 0 ? beta : 1.0f));
  } else if (at.seg <= at.last_seg) {
    // scanned: the state itself; else what the segments before this one left
    // (1 holds 0's start), the last one first decayed
    const float decay = power(beta, p.seg_tokens);
    for (int m = p.scanned || at.order == 0 ? at.order : 1; m <= at.order; ++m)
      state.add_segment(seg0 + (size_t)m * (DA * DC), tid, decay);
  }

  const uint32_t t_quad = (uint32_t)(quad * 32) << 16;
  const uint32_t t_out = tmem, t_upd = tmem + kChunk, t_state = tmem + kChunk + DA;
  const uint32_t t_low = C::kSplit ? t_upd + 64 : t_state + DA / 2;
  // The state as two 16-bit parts.  fp16 has not the range of a sum of products: they
  // are scaled by the power of two that brings the largest element to
  // 2^10 .. 2^11, and e_back undoes it.
  float e_back = 1.0f;
  auto put_state = [&](int slot) {
    float f = 1.0f;
    if constexpr (kHalf) {
      float m = 0.0f;
      state.each([&](float& e, int, int) { m = fmaxf(m, fabsf(e)); });
      const int e = max(exponent_of_all(&top[slot], m, lane, 10), -116);  // keeps 2^-e and 2^e normal
      f = power_of_2(-e);
      e_back = power_of_2(e);
    }
    constexpr int kRun = C::kSplit ? 8 : C::kCols / 4;  // pairs of neighbouring columns
#pragma unroll
    for (int rh = 0; rh < C::kRowHalves; ++rh)
#pragma unroll
      for (int j = 0; j < C::kCols / 4; j += kRun) {
        uint32_t v[kRun], rest[kRun];  // a pair's first 16 bits, and what they leave to 16 more
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
          v[i] = two_parts<T>(f * state.e[rh][2 * (j + i)], f * state.e[rh][2 * (j + i) + 1], rest[i]);
        }
        if constexpr (C::kStateTmem) {
          const uint32_t at = t_quad + ((uint32_t)(16 * rh) << 16) + half * (C::kStep / 2);
          tmem_st_pairs(t_state + at + (j ? 32 : 0), v);
          // split columns: a half's 64 side by side, in the columns it has read
          tmem_st_pairs(t_low + at + (C::kSplit ? half * (C::kStep / 2) + 2 * j : 0), rest);
        } else {  // rows of Da: 64-column boxes of DC 128-byte rows
#pragma unroll
          for (int i = 0; i < kRun; ++i) {
            const int x = half * C::kStep + 8 * (i >> 1) + (j ? 64 : 0), y = state.row + 8 * (i & 1);
            uint32_t* to = reinterpret_cast<uint32_t*>(sE + (x >> 6) * (DC * 128) + y * 128 +
                                                       ((((x & 63) >> 3) ^ (y & 7)) << 4) + (lane & 3) * 4);
            to[0] = v[i];
            to[DA * DC / 2] = rest[i];
          }
        }
      }
    if constexpr (C::kStateTmem) tmem_wait_st();
  };
  __syncwarp();
  if (n_chunks > 0) {
    put_state(0);
    gemm::fence_async_smem();
    gemm::tc_fence_before();
    __syncthreads();
  }

  const int y0 = 16 * quad + (lane >> 2);            // this lane's score rows: y0, y0 + 8
  const int tok = half * C::kToks + 2 * (lane & 3);  // its output tokens: tok + 8k (+1)
  // the third part: only the last segment's state is an output
  const bool third = !kHalf && ends;
  int fail = 0, it = 0;
  for (; it < n_chunks; ++it) {
    const uint32_t par = it & 1;
    const int t0 = at.start(it, rev);
    const int n = min(kChunk, at.len - t0);
    const bool last = ends && !rev && it == n_chunks - 1;  // leave S, not beta S
    const int ex = n - (last ? 1 : 0);
    const bool more = it + 1 < n_chunks;
    unsigned char* sB = sB2 + (it % C::kBStages) * C::kABytes;
    if (tid == 64 && more) load_b(it + 1);  // chunk it - 1 is done with its stage
    if (tid == 96) prefetch(it + 2);

    if (warp == 0) {
      if (kHalf && lane == 0) top[(it + 1) & 1] = peak[(it + 1) & 1] = most[(it + 1) & 1] = 0u;
      fail |= wait_all(bar_a, par);
      fail |= wait_all(bar_b + it % C::kBStages, (it / C::kBStages) & 1);
      gemm::tc_fence_after();
      const uint32_t e = elect_one();
      constexpr uint32_t id_s = idesc<T>(kChunk, kChunk, false, false);
      constexpr uint32_t id_x = idesc<T>(DC, kChunk, false, false);
#pragma unroll
      for (int kk = 0; kk < DA / 16; ++kk) {
        const int off = (kk / 4) * kBoxBytes + (kk % 4) * 32;
        mma_ss(e, t_upd, gemm::sdesc_sw128(sA + off), gemm::sdesc_sw128(sB + off), id_s, kk != 0);
      }
      mma_commit(e, bar_s);
#pragma unroll
      for (int part = 0; part < 2; ++part)
#pragma unroll
        for (int kk = 0; kk < DA / 16; ++kk) {
          const uint64_t q = gemm::sdesc_sw128(sA + (kk / 4) * kBoxBytes + (kk % 4) * 32);
          if constexpr (C::kStateTmem) {
            const uint32_t low = C::kSplit ? 32 * ((kk >> 1) & 1) + 16 * (kk >> 2) + 8 * (kk & 1) : 8 * kk;
            mma_ts(e, t_out, part ? t_low + low : t_state + 8 * kk, q, id_x, part | kk);
          } else {
            mma_ss(e, t_out, gemm::sdesc_sw128(sE + part * (DA * DC * 2) + (kk / 4) * (DC * 128) + (kk % 4) * 32), q,
                   id_x, part | kk);
          }
        }
      mma_commit(e, bar_x);
    }

    // decayed values in two parts, while the scores are under way
    fail |= wait_all(bar_c, par);
    if (out_f32 && it > 0) fail |= wait_all(bar_p, (it - 1) & 1);  // the last output has left sO32
    constexpr int kPieces = C::kCBytes / 16 / NT;
    float v_up = 1.0f, v_back = 1.0f;
    if constexpr (kHalf) {
      const int e = values_exponent<kPieces>(&most[par], sC, n, tid, NT);
      v_up = power_of_2(-e);
      v_back = power_of_2(e);
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int piece = i * NT + tid, y = (piece >> 3) & 63;
      uint4 high, low;
      split_piece<T>(sC, piece, y < n, decays.parts[max(0, rev ? y + 1 : ex - y)], v_up, high, low);
      reinterpret_cast<uint4*>(sW)[piece] = high;
      reinterpret_cast<uint4*>(sL)[piece] = low;
    }

    // A sum of 16-bit products may pass fp16's range where the output does not:
    // the scores are scaled by the power of two that brings the largest to
    // 2^14 .. 2^15, the inter product with them, and s_back undoes it in the
    // output.  No further up than 2^24, which leaves fp32 room for the state's part.
    float s_back = 1.0f;
    {
      // decayed scores
      fail |= wait_all(bar_s, par);
      gemm::tc_fence_after();
      float s[C::kToks / 2];
      tmem_ld_rows(t_upd + t_quad + half * C::kToks, s);
      const int x0 = half * C::kToks;
      const float* w = decays.lag + 64 + y0 - x0 - 2 * (lane & 3);
#pragma unroll
      for (int i = 0; i < C::kToks / 2; ++i) s[i] = s[i] * scale * w[8 * ((i >> 1) & 1) - 8 * (i >> 2) - (i & 1)];
      if (n < kChunk) {  // places past the sequence hold anything
#pragma unroll
        for (int i = 0; i < C::kToks / 2; ++i)
          if (max(y0 + 8 * ((i >> 1) & 1), x0 + 2 * (lane & 3) + 8 * (i >> 2) + (i & 1)) >= n) s[i] = 0.0f;
      }
      float s_scale = 1.0f;
      if constexpr (kHalf) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < C::kToks / 2; ++i) m = fmaxf(m, fabsf(s[i]));
        const int e = max(exponent_of_all(&peak[par], m, lane, 14), -24);
        s_scale = power_of_2(-e);
        s_back = power_of_2(e);
#pragma unroll
        for (int i = 0; i < C::kToks / 2; ++i) s[i] *= s_scale;
      }
      if (it > 0) fail |= wait_all(bar_p, (it - 1) & 1);  // the last output has left sP
      auto at_score = [&](unsigned char* tile, int k) {  // and 1024 bytes on: row y0 + 8
        return reinterpret_cast<uint32_t*>(tile + y0 * 128 + ((((x0 >> 3) + k) ^ (y0 & 7)) << 4) + (lane & 3) * 4);
      };
      uint32_t rest[C::kToks / 4];  // what the first 16 bits leave, to 16 more
#pragma unroll
      for (int i = 0; i < C::kToks / 4; ++i)
        at_score(sP, i >> 1)[(i & 1) * 256] = two_parts<T>(s[2 * i], s[2 * i + 1], rest[i]);
      fail |= wait_all(bar_x, par);
      gemm::tc_fence_after();
#pragma unroll
      for (int i = 0; i < C::kToks / 4; ++i) at_score(sQ, i >> 1)[(i & 1) * 256] = rest[i];
      if (tid == 32 && more && !third) load_a(it + 1);
      __syncwarp();
      // the inter product, decayed, is what the intra product adds to
      float f[C::kToks / 4];
#pragma unroll
      for (int i = 0; i < C::kToks / 4; ++i) {
        const int y = tok + 8 * (i >> 1) + (i & 1);
        f[i] = s_scale * e_back * scale * decays.lag[64 + (rev ? y + 1 - n : y)];
      }
#pragma unroll
      for (int rh = 0; rh < C::kRowHalves; ++rh) {
        float x[C::kToks / 2];
        const uint32_t at = t_out + t_quad + ((uint32_t)(16 * rh) << 16) + half * C::kToks;
        tmem_ld_rows(at, x);
#pragma unroll
        for (int i = 0; i < C::kToks / 2; ++i) x[i] *= f[2 * (i >> 2) + (i & 1)];
        tmem_st_rows(at, x);
      }
    }
    if (third) {  // where a was: the scores and the inter product have read it
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int piece = i * NT + tid, y = (piece >> 3) & 63;
        reinterpret_cast<uint4*>(sA)[piece] =
            third_part<T>(sC, piece, y < n, decays.of(max(0, rev ? y + 1 : ex - y), rev),
                          reinterpret_cast<const uint4*>(sW)[piece],
                          reinterpret_cast<const uint4*>(sL)[piece]);
      }
    }
    if (n < kChunk) {
      clear_rows(sB, C::kABytes, n, tid, NT);
      clear_rows(sC, C::kCBytes, n, tid, NT);
    }
    gemm::fence_async_smem();
    gemm::tc_fence_before();
    if (__syncthreads_or(fail)) break;

    auto update = [&](uint32_t e, const unsigned char* values, uint32_t accumulate) {
      constexpr uint32_t id = idesc<T>(DC, DA, true, true);
#pragma unroll
      for (int kk = 0; kk < kChunk / 16; ++kk)
        mma_ss(e, t_upd, sdesc_mn(values + kk * 2048, kBoxBytes), sdesc_mn(sB + kk * 2048, kBoxBytes), id,
               accumulate | (kk != 0));
    };
    if (warp == 0) {
      gemm::tc_fence_after();
      const uint32_t e = elect_one();
      constexpr uint32_t id = idesc<T>(DC, kChunk, true, false);
#pragma unroll
      for (int kk = 0; kk < kChunk / 8; ++kk)
        mma_ss(e, t_out, sdesc_mn(sC + (kk & 3) * 2048, kBoxBytes),
               gemm::sdesc_sw128((kk < 4 ? sP : sQ) + (kk & 3) * 32), id, 1);
      mma_commit(e, bar_o);
      update(e, sW, 0);
      update(e, sL, 1);
      if (third) update(e, sA, 1);
      mma_commit(e, bar_u);
    }

    fail |= wait_all(bar_o, par);
    gemm::tc_fence_after();
    if (tid == 96 && more) load_c(it + 1);
    __syncwarp();
    auto output = [&](auto put) {  // put(16-lane half, its registers)
#pragma unroll
      for (int rh = 0; rh < C::kRowHalves; ++rh) {
        float o[C::kToks / 2];
        tmem_ld_rows(t_out + t_quad + ((uint32_t)(16 * rh) << 16) + half * C::kToks, o);
        if constexpr (kHalf) {
#pragma unroll
          for (int i = 0; i < C::kToks / 2; ++i) o[i] *= s_back;
        }
        if (n < kChunk) {
#pragma unroll
          for (int i = 0; i < C::kToks / 2; ++i)
            if (tok + 8 * (i >> 2) + (i & 1) >= n) o[i] = 0.0f;
        }
        put(rh, o);
      }
    };
    if (!out_f32) {
      output([&](int rh, const float (&o)[C::kToks / 2]) {
        // tokens as rows again: blocks (channels, +8) x (tokens 16j, 16j + 8)
        const int x = (state.row - (lane >> 2)) + 16 * rh;  // the warp's first channel
        unsigned char* tile = sP + (x >> 6) * kBoxBytes;
#pragma unroll
        for (int j = 0; j < C::kToks / 16; ++j) {
          const int y = half * C::kToks + 16 * j + 8 * (lane >> 4) + (lane & 7);
          const int piece = ((x & 63) >> 3) + ((lane >> 3) & 1);
          stmatrix_t(tile + y * 128 + ((piece ^ (y & 7)) << 4),
                     Elem<T>::from2(o[8 * j], o[8 * j + 1]), Elem<T>::from2(o[8 * j + 2], o[8 * j + 3]),
                     Elem<T>::from2(o[8 * j + 4], o[8 * j + 5]), Elem<T>::from2(o[8 * j + 6], o[8 * j + 7]));
        }
      });
    }

    fail |= wait_all(bar_u, par);
    gemm::tc_fence_after();
    if (out_f32) {
      output([&](int rh, const float (&o)[C::kToks / 2]) {  // boxes of 32 channels (128 bytes) x 64 tokens
#pragma unroll
        for (int i = 0; i < C::kToks / 2; ++i) {
          const int x = state.row + 16 * rh + 8 * ((i >> 1) & 1), y = tok + 8 * (i >> 2) + (i & 1);
          *reinterpret_cast<float*>(sO32 + (x >> 5) * kBoxBytes + y * 128 + ((((x & 31) >> 2) ^ (y & 7)) << 4) +
                                    (x & 3) * 4) = o[i];
        }
      });
    }
    if (tid == 32 && more && third) load_a(it + 1);
    __syncwarp();
    state.add_update(t_upd + t_quad + half * C::kStep, decays.of(ex, rev), v_back);
    if (more) put_state((it + 1) & 1);
    gemm::fence_async_smem();
    gemm::tc_fence_before();
    if (__syncthreads_or(fail)) break;
    if (tid == kStorer) {
      if (out_f32) {
#pragma unroll 1
        for (int x = 0; x < Dc; x += 32) tma_store_4d(&maps.out, sO32 + (x >> 5) * kBoxBytes, x, t0, ho, b);
      } else {
#pragma unroll
        for (int x = 0; x < DC / 64; ++x)
          if (64 * x < Dc) tma_store_4d(&maps.out, sP + x * kBoxBytes, 64 * x, t0, ho, b);
      }
      gemm::bulk_commit();
      bulk_wait_read_all();
      mbar_arrive(bar_p);
    }
  }
  if (it < n_chunks) {  // a wait gave up
    if (fail) record_status(g.status, kStatusTimeout);
    // loads in flight land before the block may exit: chunk it's, and chunk
    // it + 1's where they were started
    if (tid == 0) {
      for (int j = it; j < it + 2; ++j) {
        mbar_wait_bounded(bar_a, j & 1, gemm::kDrainWaitNs / 4);
        mbar_wait_bounded(bar_b + j % C::kBStages, (j / C::kBStages) & 1, gemm::kDrainWaitNs / 4);
        mbar_wait_bounded(bar_c, j & 1, gemm::kDrainWaitNs / 4);
      }
    }
  } else if (ends) {
    state.store(g, r, b, h, rev ? scale : 1.0f);
  }
  {
    // whole chunks past the sequence's end
    const int from = at.begin + at.chunks * kChunk;
    const int to = min(T_all, at.begin + p.seg_tokens);
    const int per = out_f32 ? 4 : 8, pieces = Dc / per;
    const size_t es = out_f32 ? 4 : 2;
    unsigned char* o = static_cast<unsigned char*>(r.out.data) + (b * r.out.sb + ho * r.out.sh) * es;
    for (int i = tid; i < (to - from) * pieces; i += NT)
      *reinterpret_cast<uint4*>(o + ((from + i / pieces) * r.out.st + (i % pieces) * per) * es) =
          make_uint4(0, 0, 0, 0);
  }
  if (tid == kStorer) gemm::bulk_wait_all();
  gemm::tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    gemm::tc_fence_after();
    gemm::tmem_dealloc(tmem, C::kTmemCols);
  }
}

}  // namespace attn
}  // namespace snn
