// Block norms: the norm after a block, its gate and residual scale, the
// residual sum and the norm before the next block, per row of N channels:
//   n  = a rstd_a w_post            rstd_a = rsqrt(mean over the group of a^2 + eps)
//   r' = r + s n act(z)
//   y  = r' rstd w_pre              rstd   = rsqrt(mean over the row of r'^2 + eps)
// and the gradients (g = grad_y w_pre, e = r' rstd):
//   d      = grad_r' + rstd (g - e mean(g e))
//   grad_r = d;  grad_z = d s n act'(z)
//   grad_a = rstd_a (m - h mean_group(m h)),  h = a rstd_a,  m = d s act(z) w_post
//   grad_w_post = s G,  grad_s = w_post G  with  G = sum d act(z) h;  grad_w_pre = sum grad_y e
// Every tensor is read and written once: the bound is HBM.  One warp (short
// rows) or one block takes a row, eight channels to a thread; blocks stay on the
// GPU and take rows in turn, with the next row or two on their way to shared
// memory (16-byte asynchronous copies) while the present one is worked on.  Rows of
// whole 16-byte vectors are copied and read by the thread that owns the
// channels; rows of any other length or stride are copied as the aligned
// vectors that cover them and read element by element.  The parameters' gradients gather in the registers (long
// rows: in shared memory) of the thread that owns the channels over all the
// rows of its block, so the sums over rows need one [blocks, 2, N] array of
// partials and a second kernel that adds them in block order (no atomics: the
// same bits on every call).
//
// Arithmetic is on pairs of channels (f32x2): rows of 16-bit values are bound by
// instruction issue as much as by HBM (one channel an instruction: 16384 x 2048
// bf16 68 us forward, 119 backward).
//
// Measured (share of the copy rate): forward of 16384 x 4096, 16-bit on a 32-bit
// stream, 151 us (0.92); of 16384 x 2048 bf16 58 us (0.85); of 8192 x 8192 bf16
// 137 us (0.72); of 2000 x 7049 on a 32-bit stream, element by element, 52 us
// (0.56).  Backward of 8192 x 4096 on a 32-bit stream 128 us (0.85); of 16384 x
// 2048 bf16 with a norm per head 104 us (0.76); of 3001 x 1001 fp32 25 us (0.57);
// of 4096 x 8192 bf16 189 us (0.42: one block of 1024 threads on an SM, nothing
// beside its barriers, sums and parameters outside its registers).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "launch.cuh"
#include "scan_host.cuh"
#include "snn.h"
#include "snn_device.cuh"

namespace snn {
namespace norm {

constexpr int64_t kMaxN = 8192;
constexpr int kSms = 152;
constexpr int E = 8;  // channels of a thread
constexpr int kBwdThreads = 512;  // of the backward's blocks on an SM

struct Rows {
  void* data;
  int64_t ld;
};

struct Args {
  int64_t M;
  int N, group, gate;
  float eps;
  Rows r, a, z, ro, y;        // forward
  Rows gro, gy, gr, ga, gz;   // backward (reads ro, a, z)
  const float *w_post, *scale, *w_pre;
  int stages;                 // rows a team has in shared memory at once, 1 to 3
  float* part;                // [blocks][2][N]
};

// Two channels an instruction: fma, mul and add of a pair of floats, each half
// rounded as by itself.
__device__ __forceinline__ uint64_t bits(float2 a) {
  uint64_t w;
  asm("mov.b64 %0, {%1, %2};" : "=l"(w) : "f"(a.x), "f"(a.y));
  return w;
}
__device__ __forceinline__ float2 halves(uint64_t w) {
  float2 a;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a.x), "=f"(a.y) : "l"(w));
  return a;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t w;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(w) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
  return halves(w);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t w;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(w) : "l"(bits(a)), "l"(bits(b)));
  return halves(w);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t w;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(w) : "l"(bits(a)), "l"(bits(b)));
  return halves(w);
}
__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }
__device__ __forceinline__ float2 two(const float* v, int e) { return make_float2(v[e], v[e + 1]); }
__device__ __forceinline__ void put2(float* v, int e, float2 a) {
  v[e] = a.x;
  v[e + 1] = a.y;
}

// 1 / (1 + e^-z) of two channels, for gates of type T.  16-bit ones take the
// approximate power of two and reciprocal: the rounding of z log2(e) costs up to
// |z| 2^-24 of the result (5e-6 at most, a hundredth of fp16's half unit), and below
// about -87 it is zero.
template <typename T>
__device__ __forceinline__ float2 sigmoid2(float2 z) {
  if constexpr (sizeof(T) == 4)
    return make_float2(__frcp_rn(1.0f + expf(-z.x)), __frcp_rn(1.0f + expf(-z.y)));
  constexpr float kLog2E = 1.44269504088896340736f;
  float2 p = mul2(z, both(-kLog2E));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(p.x));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(p.y));
  p = add2(p, both(1.0f));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(p.x));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(p.y));
  return p;
}

// Eight floats as one 32-byte access: two 16-byte ones would each touch half of
// every 32-byte sector (norms of 16384x4096 on a 32-bit stream: 168 us, 210 with
// halves).  A matrix that starts between 32-byte boundaries takes the halves.
__device__ __forceinline__ bool wide(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0; }
__device__ __forceinline__ void store32(float* p, const float v[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]),
               "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}

// 16 bytes from global to shared memory, both aligned.
__device__ __forceinline__ void copy16(unsigned char* dst, const unsigned char* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
// (by the whole warp at once: its copies are counted together)
__device__ __forceinline__ void copies_commit() {
  __syncwarp();
  asm volatile("cp.async.commit_group;" ::: "memory");
}
__device__ __forceinline__ void copies_wait(int left) {  // all groups of this thread but the newest
  if (left == 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
  else if (left == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 2;" ::: "memory");
}

// Bytes a row of a tensor takes in shared memory (16 more for a row that does
// not start on a 16-byte boundary).
__host__ __device__ constexpr int slot_bytes(int N, int size) { return (N * size + 15) / 16 * 16 + 16; }

// One tensor's row in shared memory; a thread's share is eight consecutive
// channels (VEC), else every TPR-th.
template <typename T, bool VEC, int TPR>
struct Slot {
  unsigned char* smem;

  __device__ __forceinline__ static const unsigned char* row_of(const Rows& m, int64_t row) {
    return reinterpret_cast<const unsigned char*>(static_cast<const T*>(m.data) + row * m.ld);
  }
  __device__ __forceinline__ void fetch(const Rows& m, int64_t row, int64_t M, int N, int t) const {
    const unsigned char* src = row_of(m, row);
    if constexpr (VEC) {
      if (t * E >= N) return;
#pragma unroll
      for (int i = 0; i < E * (int)sizeof(T) / 16; ++i) {
        const int o = t * E * (int)sizeof(T) + 16 * i;
        copy16(smem + o, src + o);
      }
    } else {
      const int skew = (int)(reinterpret_cast<uintptr_t>(src) & 15u), end = skew + N * (int)sizeof(T);
      // whole vectors as far as the matrix goes: past the row's end lies the next row
      const int64_t rest = skew + ((M - 1 - row) * m.ld + N) * (int64_t)sizeof(T);
#pragma unroll
      for (int k = 0; k <= E * (int)sizeof(T) / 16; ++k) {
        const int o = 16 * (k * TPR + t);
        if (o + 16 <= rest && o < end) {
          copy16(smem + o, src - skew + o);
        } else if (o < end) {  // the matrix's last elements
          for (int i = o; i < end; i += (int)sizeof(T))
            if (i >= skew) *reinterpret_cast<T*>(smem + i) = *reinterpret_cast<const T*>(src - skew + i);
        }
      }
    }
  }
  // in 32 bits, zero past N
  __device__ __forceinline__ void get(const Rows& m, int64_t row, int N, int t, float v[E]) const {
    if constexpr (VEC) {
      if (t * E < N) {
        Elem<T>::load8(reinterpret_cast<const T*>(smem) + t * E, v);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = 0.0f;
      }
    } else {
      const int skew = (int)(reinterpret_cast<uintptr_t>(row_of(m, row)) & 15u);
      const T* x = reinterpret_cast<const T*>(smem + skew);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = e * TPR + t < N ? (float)x[e * TPR + t] : 0.0f;
    }
  }
};

// A thread's eight consecutive channels of a row, as they lie in memory, in
// registers.
__device__ __forceinline__ void load32(const float* p, uint4 w[2]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0].x), "=r"(w[0].y), "=r"(w[0].z), "=r"(w[0].w), "=r"(w[1].x), "=r"(w[1].y),
                 "=r"(w[1].z), "=r"(w[1].w)
               : "l"(p)
               : "memory");
}
template <typename T>
struct Held {
  uint4 w[E * sizeof(T) / 16];
  __device__ __forceinline__ void fetch(const Rows& m, int64_t row, int N, int t) {
    const T* p = static_cast<const T*>(m.data) + row * m.ld + t * E;
    if (t * E >= N) return;
    if (sizeof(T) == 4 && wide(p)) {
      load32(reinterpret_cast<const float*>(p), w);
    } else {
#pragma unroll
      for (int i = 0; i < (int)(E * sizeof(T) / 16); ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
    }
  }
  __device__ __forceinline__ void get(int N, int t, float v[E]) const {
    if (t * E < N) {
      Elem<T>::load8(reinterpret_cast<const T*>(w), v);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = 0.0f;
    }
  }
};

template <typename T, bool VEC, int TPR>
__device__ __forceinline__ void store_row(const Rows& m, int64_t row, int N, int t, const float v[E]) {
  T* p = static_cast<T*>(m.data) + row * m.ld;
  if constexpr (VEC) {
    if (t * E < N) {
      if constexpr (sizeof(T) == 4) {
        if (wide(p)) store32(p + t * E, v);
        else Elem<T>::store8(p + t * E, v);
      } else {
        Elem<T>::store8(p + t * E, v);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e * TPR + t < N) Elem<T>::store1(p + e * TPR + t, v[e]);
  }
}

// A parameter's share (ones where it is absent, zero past N).
template <bool VEC, int TPR>
__device__ __forceinline__ void load_param(const float* p, int N, int t, float v[E]) {
  if (VEC && p && t * E < N) {
    Elem<float>::load8(p + t * E, v);
    return;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int c = VEC ? t * E + e : e * TPR + t;
    v[e] = c < N ? (p ? p[c] : 1.0f) : 0.0f;
  }
}

// Sums of K values over the TPR threads of a row; every thread gets them.
// Successive sums alternate between two scratch buffers, so one barrier a sum
// is enough: a warp cannot be two sums ahead.
template <int TPR>
struct RowSum {
  float (*scratch)[3][32];  // [2][value][warp]
  int turn = 0;
  // in_group: the last value's sum over a group's `lanes` neighbouring threads
  template <int K>
  __device__ __forceinline__ void operator()(float (&v)[K], int lanes = 32, float* in_group = nullptr) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      if (in_group && o == lanes) *in_group = v[K - 1];
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
    if (in_group && lanes >= 32) *in_group = v[K - 1];
    if constexpr (TPR > 32) {
      constexpr int W = TPR / 32;
      float (*s)[32] = scratch[turn];
      turn ^= 1;
      if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) s[k][threadIdx.x >> 5] = v[k];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) {
        float2 a = make_float2(s[k][0], s[k][1]);
#pragma unroll
        for (int w = 0; w + 4 <= W; w += 4) {
          const float4 x = *reinterpret_cast<const float4*>(&s[k][w]);
          const float2 lo = make_float2(x.x, x.y), hi = make_float2(x.z, x.w);
          a = w ? add2(a, add2(lo, hi)) : add2(lo, hi);
        }
        v[k] = a.x + a.y;
      }
    }
  }
};

// Sum of a b over a thread's channels, and of a^2.
__device__ __forceinline__ float dot(const float a[E], const float b[E]) {
  float2 s = mul2(two(a, 0), two(b, 0));
#pragma unroll
  for (int e = 2; e < E; e += 2) s = fma2(two(a, e), two(b, e), s);
  return s.x + s.y;
}
__device__ __forceinline__ float square_sum(const float a[E]) { return dot(a, a); }

// Sum over the group of `lanes` neighbouring threads that a vector lies in.
__device__ __forceinline__ float group_sum(float v, int lanes) {
  for (int o = 1; o < lanes; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <int TPR>
constexpr int kBlockThreads = TPR == 32 ? 256 : TPR;  // short rows: eight warps, a row each
template <int TPR>
constexpr int kTeams = kBlockThreads<TPR> / TPR;

// Before a team reads what its other threads copied.
template <int TPR>
__device__ __forceinline__ void team_sync() {
  if constexpr (TPR == 32) __syncwarp();
  else __syncthreads();
}

// Shared memory of a stage: the rows a team reads.
__host__ __device__ constexpr int fwd_stage(int N, int t_size, int r_size) {
  return slot_bytes(N, r_size) + 2 * slot_bytes(N, t_size);
}
__host__ __device__ constexpr int bwd_stage(int N, int t_size, int r_size) {
  return 2 * slot_bytes(N, r_size) + 3 * slot_bytes(N, t_size);
}

extern __shared__ __align__(16) unsigned char norm_smem[];

template <typename T, typename R, bool VEC, int TPR>
__global__ void __launch_bounds__(kBlockThreads<TPR>, 1024 / kBlockThreads<TPR>) norm_fwd(const Args g) {
  __shared__ __align__(16) float scratch[2][3][32];
  grid_dep_wait();
  const int t = threadIdx.x % TPR, team = threadIdx.x / TPR, N = g.N;
  const int64_t step = (int64_t)gridDim.x * kTeams<TPR>;
  int64_t row = (int64_t)blockIdx.x * kTeams<TPR> + team;
  const bool whole = g.group == N, block = g.a.data != nullptr, gated = g.z.data != nullptr;
  const bool silu = g.gate == SNN_GATE_SILU;
  const float inv_n = 1.0f / (float)N, inv_g = 1.0f / (float)g.group;
  RowSum<TPR> row_sum{scratch};
  float w_post[E], w_pre[E];
  load_param<VEC, TPR>(g.w_pre, N, t, w_pre);
  if (block) {  // s n act(z): the two factors of a channel as one
    float sc[E];
    load_param<VEC, TPR>(g.w_post, N, t, w_post);
    load_param<VEC, TPR>(g.scale, N, t, sc);
#pragma unroll
    for (int e = 0; e < E; ++e) w_post[e] *= sc[e];
  }
  const int stage = fwd_stage(N, sizeof(T), sizeof(R));
  unsigned char* const base = norm_smem + team * g.stages * stage;
  auto r_slot = [&](int k) { return Slot<R, VEC, TPR>{base + k * stage}; };
  auto a_slot = [&](int k) { return Slot<T, VEC, TPR>{base + k * stage + slot_bytes(N, sizeof(R))}; };
  auto z_slot = [&](int k) {
    return Slot<T, VEC, TPR>{base + k * stage + slot_bytes(N, sizeof(R)) + slot_bytes(N, sizeof(T))};
  };
  auto fetch = [&](int64_t i, int k) {
    if (i < g.M) {
      r_slot(k).fetch(g.r, i, g.M, N, t);
      if (block) a_slot(k).fetch(g.a, i, g.M, N, t);
      if (gated) z_slot(k).fetch(g.z, i, g.M, N, t);
    }
    copies_commit();
  };
  const int ahead = g.stages - 1;  // at least one
  for (int i = 0; i < ahead; ++i) fetch(row + i * step, i);
  for (int k = 0, next = ahead; row < g.M; row += step) {
    fetch(row + ahead * step, next);  // that stage was read before the last row's sums
    copies_wait(ahead);
    if (!VEC) team_sync<TPR>();
    float x[E], u[E];
    r_slot(k).get(g.r, row, N, t, x);
    if (block) {
      a_slot(k).get(g.a, row, N, t, u);
      float ss[1] = {square_sum(u)};
      if (whole) row_sum(ss);
      else ss[0] = group_sum(ss[0], g.group >> 3);
      const float rstd = rsqrtf(fmaf(ss[0], whole ? inv_n : inv_g, g.eps));
      float z[E];
      if (gated) z_slot(k).get(g.z, row, N, t, z);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 n = mul2(mul2(two(u, e), both(rstd)), two(w_post, e));
        float2 act = both(1.0f);
        if (gated) {
          act = sigmoid2<T>(two(z, e));
          if (silu) act = mul2(act, two(z, e));
        }
        put2(x, e, fma2(n, act, two(x, e)));
      }
      store_row<R, VEC, TPR>(g.ro, row, N, t, x);
    }
    float ss[1] = {square_sum(x)};
    row_sum(ss);  // also where there is no y: it is what frees the stage
    if (TPR == 32) team_sync<TPR>();
    if (g.y.data) {
      const float rstd = rsqrtf(fmaf(ss[0], inv_n, g.eps));
#pragma unroll
      for (int e = 0; e < E; e += 2) put2(x, e, mul2(mul2(two(x, e), both(rstd)), two(w_pre, e)));
      store_row<T, VEC, TPR>(g.y, row, N, t, x);
    }
    k = k + 1 == g.stages ? 0 : k + 1;
    next = next + 1 == g.stages ? 0 : next + 1;
  }
  copies_wait(0);
}

// Two vectors of a thread's channels: parameters, or sums over rows.  In
// registers; for long rows, whose threads have none to spare, the sums lie in
// shared memory ([2][E / 4][threads] float4) and the parameters are read again.
template <bool SMEM>
struct Sums {
  float v[SMEM ? 1 : 2][E];
  float4* at;
  int threads;
  __device__ __forceinline__ float4& word(int k, int i) { return at[(k * (E / 4) + i) * threads + threadIdx.x]; }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if constexpr (SMEM) {
#pragma unroll
        for (int i = 0; i < E / 4; ++i) word(k, i) = make_float4(0.f, 0.f, 0.f, 0.f);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[k][e] = 0.0f;
      }
    }
  }
  __device__ __forceinline__ void get(int k, float (&a)[E]) {
    if constexpr (SMEM) {
#pragma unroll
      for (int i = 0; i < E / 4; ++i) {
        const float4 s = word(k, i);
        a[4 * i] = s.x;
        a[4 * i + 1] = s.y;
        a[4 * i + 2] = s.z;
        a[4 * i + 3] = s.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) a[e] = v[k][e];
    }
  }
  __device__ __forceinline__ void add(int k, const float (&a)[E], const float (&b)[E]) {  // += a b
    if constexpr (SMEM) {
#pragma unroll
      for (int i = 0; i < E / 4; ++i) {
        float4 s = word(k, i);
        s.x = fmaf(a[4 * i], b[4 * i], s.x);
        s.y = fmaf(a[4 * i + 1], b[4 * i + 1], s.y);
        s.z = fmaf(a[4 * i + 2], b[4 * i + 2], s.z);
        s.w = fmaf(a[4 * i + 3], b[4 * i + 3], s.w);
        word(k, i) = s;
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; e += 2) put2(v[k], e, fma2(two(a, e), two(b, e), two(v[k], e)));
    }
  }
};

template <typename T, typename R, bool VEC, int TPR>
__global__ void __launch_bounds__(kBlockThreads<TPR>, TPR == 1024 ? 1 : kBwdThreads / kBlockThreads<TPR>)
    norm_bwd(const Args g) {
  __shared__ __align__(16) float scratch[2][3][32];
  grid_dep_wait();
  // Five tensors' next row in registers rather than in shared memory, where the
  // threads have them: whole vectors of rows up to 4096 channels (8192 rows of
  // 4096, 16-bit on a 32-bit stream: 129 us, 151 through shared memory).
  constexpr bool kLong = TPR == 1024, kHeld = VEC && !kLong;
  const int t = threadIdx.x % TPR, team = threadIdx.x / TPR, N = g.N;
  const int64_t step = (int64_t)gridDim.x * kTeams<TPR>;
  int64_t row = (int64_t)blockIdx.x * kTeams<TPR> + team;
  const bool whole = !VEC || g.group == N, block = g.a.data != nullptr, gated = g.z.data != nullptr;
  const bool silu = g.gate == SNN_GATE_SILU;
  const bool pre = g.gy.data != nullptr, through = g.gro.data != nullptr;
  const float inv_n = 1.0f / (float)N, inv_g = 1.0f / (float)g.group;
  RowSum<TPR> row_sum{scratch};
  const int stage = bwd_stage(N, sizeof(T), sizeof(R));
  unsigned char* const base = norm_smem + team * g.stages * stage;
  const int r_bytes = slot_bytes(N, sizeof(R)), t_bytes = slot_bytes(N, sizeof(T));
  auto ro_slot = [&](int k) { return Slot<R, VEC, TPR>{base + k * stage}; };
  auto gro_slot = [&](int k) { return Slot<R, VEC, TPR>{base + k * stage + r_bytes}; };
  auto t_slot = [&](int k, int i) { return Slot<T, VEC, TPR>{base + k * stage + 2 * r_bytes + i * t_bytes}; };
  auto fetch = [&](int64_t i, int k) {
    if (i < g.M) {
      if (pre) ro_slot(k).fetch(g.ro, i, g.M, N, t);
      if (pre) t_slot(k, 0).fetch(g.gy, i, g.M, N, t);
      if (through) gro_slot(k).fetch(g.gro, i, g.M, N, t);
      if (block) t_slot(k, 1).fetch(g.a, i, g.M, N, t);
      if (gated) t_slot(k, 2).fetch(g.z, i, g.M, N, t);
    }
    copies_commit();
  };
  const int ahead = g.stages - 1;
  Held<R> held_ro, held_gro;
  Held<T> held_gy, held_a, held_z;
  auto hold = [&](int64_t i) {
    if (i >= g.M) return;
    if (pre) held_ro.fetch(g.ro, i, N, t);
    if (pre) held_gy.fetch(g.gy, i, N, t);
    if (through) held_gro.fetch(g.gro, i, N, t);
    if (block) held_a.fetch(g.a, i, N, t);
    if (gated) held_z.fetch(g.z, i, N, t);
  };
  if constexpr (kHeld) {
    hold(row);
  } else {
    for (int i = 0; i < (ahead ? ahead : 1); ++i) fetch(row + i * step, i);
  }
  Sums<kLong> sums;  // 0: of d act(z) h, 1: of grad_y y'
  sums.at = reinterpret_cast<float4*>(norm_smem + g.stages * stage);
  sums.threads = TPR;
  sums.clear();
  float w_pre[E], c[E];  // c: the factors s w_post of a channel as one
  auto params = [&]() {
    float sc[E];
    load_param<VEC, TPR>(g.w_pre, N, t, w_pre);
    load_param<VEC, TPR>(g.w_post, N, t, c);
    load_param<VEC, TPR>(g.scale, N, t, sc);
#pragma unroll
    for (int e = 0; e < E; ++e) c[e] *= sc[e];
  };
  if (!kLong) params();
  for (int k = 0, next = ahead; row < g.M; row += step) {
    float d[E], x[E], gw[E], h[E], z_held[kHeld ? E : 1];
    float* const z = kHeld ? z_held : gw;  // read late into grad_y's place, or held
    if constexpr (kHeld) {
      if (pre) held_ro.get(N, t, x);
      if (pre) held_gy.get(N, t, gw);
      if (through) held_gro.get(N, t, d);
      if (block) held_a.get(N, t, h);
      if (gated) held_z.get(N, t, z);
      hold(row + step);
    } else {
      if (ahead) fetch(row + ahead * step, next);  // that stage was read before the last row's sums
      copies_wait(ahead);
      if (!VEC) team_sync<TPR>();
      if (pre) ro_slot(k).get(g.ro, row, N, t, x);
      if (pre) t_slot(k, 0).get(g.gy, row, N, t, gw);
      if (block) t_slot(k, 1).get(g.a, row, N, t, h);
    }
    if (kLong) load_param<VEC, TPR>(g.w_pre, N, t, w_pre);
    float ss[3] = {0.0f, 0.0f, 0.0f};  // of r'^2, grad_y w_pre r', a^2
    if (pre) {
      float v[E];
#pragma unroll
      for (int e = 0; e < E; e += 2) put2(v, e, mul2(two(gw, e), two(w_pre, e)));
      ss[0] = square_sum(x);
      ss[1] = dot(v, x);
    }
    if (block) ss[2] = square_sum(h);
    float in_group = 0.0f;
    if (kHeld && !whole) {
      row_sum(ss, g.group >> 3, &in_group);
    } else {
      if (kLong && block && !whole) in_group = group_sum(ss[2], g.group >> 3);
      row_sum(ss);
    }
    if (!through) {
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = 0.0f;
    } else if (!kHeld) {
      gro_slot(k).get(g.gro, row, N, t, d);
    }
    if (pre) {
      const float rstd = rsqrtf(fmaf(ss[0], inv_n, g.eps));
      const float mean = ss[1] * rstd * inv_n;  // mean of (grad_y w_pre) y'
#pragma unroll
      for (int e = 0; e < E; e += 2) put2(x, e, mul2(two(x, e), both(rstd)));  // y'
      sums.add(1, gw, x);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 v = fma2(two(x, e), both(-mean), mul2(two(gw, e), two(w_pre, e)));
        put2(d, e, fma2(both(rstd), v, two(d, e)));
      }
    }
    if (g.gr.data) store_row<R, VEC, TPR>(g.gr, row, N, t, d);
    float q[1] = {0.0f};
    const float rstd_a = rsqrtf(whole ? fmaf(ss[2], inv_n, g.eps) : fmaf(in_group, inv_g, g.eps));
    if (block) {
      if (kLong) params();
      if (!kHeld && gated) t_slot(k, 2).get(g.z, row, N, t, z);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 hn = mul2(two(h, e), both(rstd_a)), dr = two(d, e);
        float2 m = mul2(dr, two(c, e));
        put2(h, e, hn);
        put2(x, e, dr);
        if (gated) {
          const float2 s = sigmoid2<T>(two(z, e)), rest = fma2(s, both(-1.0f), both(1.0f));
          float2 act = s, slope = mul2(s, rest);
          if (silu) {
            act = mul2(two(z, e), s);
            slope = fma2(act, rest, s);
          }
          put2(z, e, mul2(mul2(m, hn), slope));  // grad_z
          put2(x, e, mul2(dr, act));
          m = mul2(m, act);
        }
        put2(d, e, m);
      }
      q[0] = dot(d, h);
      sums.add(0, x, h);
      if (g.gz.data) store_row<T, VEC, TPR>(g.gz, row, N, t, z);
    }
    // the row is read (VEC: by the threads that copied it): its stage is free
    if (whole) row_sum(q);
    else if (block) q[0] = group_sum(q[0], g.group >> 3);
    if (!VEC && TPR == 32) team_sync<TPR>();
    if (!kHeld && !ahead) fetch(row + step, 0);
    if (g.ga.data) {
      const float mean = q[0] * (whole ? inv_n : inv_g);
#pragma unroll
      for (int e = 0; e < E; e += 2)
        put2(d, e, mul2(both(rstd_a), fma2(two(h, e), both(-mean), two(d, e))));
      store_row<T, VEC, TPR>(g.ga, row, N, t, d);
    }
    k = k + 1 == g.stages ? 0 : k + 1;
    next = next + 1 == g.stages ? 0 : next + 1;
  }
  copies_wait(0);
  if (!g.part) return;
  float* p = g.part + (int64_t)blockIdx.x * 2 * N;
  if constexpr (kTeams<TPR> > 1) {  // the block's teams, in order
    constexpr int kWidth = TPR * E;
    float* all = reinterpret_cast<float*>(norm_smem);  // [teams][2][kWidth], over the rows
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float v[E];
      sums.get(k, v);
#pragma unroll
      for (int e = 0; e < E; ++e) all[(team * 2 + k) * kWidth + (VEC ? t * E + e : e * TPR + t)] = v[e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * N; i += kBlockThreads<TPR>) {
      const int k = i / N, at = k * kWidth + i - k * N;
      float v = all[at];
#pragma unroll
      for (int j = 1; j < kTeams<TPR>; ++j) v += all[j * 2 * kWidth + at];
      p[i] = v;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float v[E];
      sums.get(k, v);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int at = VEC ? t * E + e : e * TPR + t;
        if (at < N) p[k * N + at] = v[e];
      }
    }
  }
}

// Column sums of the partials: 32 columns a block, the rows in 32 slices (every
// 32nd row, in order), then the slices in order.
__global__ void __launch_bounds__(1024) norm_sum(const float* __restrict__ part, int rows, int N,
                                                 const float* w_post, const float* scale,
                                                 float* g_post, float* g_scale, float* g_pre) {
  __shared__ float s[32][33];
  grid_dep_wait();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31);
  const int slice = threadIdx.x >> 5, width = 2 * N;
  float v = 0.0f;
  if (c < width) {
#pragma unroll 4
    for (int i = slice; i < rows; i += 32) v += part[(int64_t)i * width + c];
  }
  s[slice][threadIdx.x & 31] = v;
  __syncthreads();
  if (slice || c >= width) return;
  for (int i = 1; i < 32; ++i) v += s[i][threadIdx.x];
  if (c >= N) {
    if (g_pre) g_pre[c - N] = v;
  } else {
    if (g_post) g_post[c] = scale ? scale[c] * v : v;
    if (g_scale) g_scale[c] = w_post ? w_post[c] * v : v;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

// Threads of a row, eight channels each.
int row_threads(int64_t N) {
  return N <= 256 ? 32 : N <= 512 ? 64 : N <= 1024 ? 128 : N <= 2048 ? 256 : N <= 4096 ? 512 : 1024;
}

// Blocks for M rows with `threads` of them on an SM; from the shape alone, so
// that a shape always sums in the same order.
int64_t blocks_for(int64_t M, int64_t N, int threads) {
  const int tpr = row_threads(N), block = tpr == 32 ? 256 : tpr;
  const int64_t resident = (int64_t)kSms * (threads > block ? threads / block : 1);
  return least(resident, tpr == 32 ? (M + 7) / 8 : M);
}
int64_t bwd_blocks(int64_t M, int64_t N) { return blocks_for(M, N, kBwdThreads); }

snn_status_t check_desc(const snn_norm_desc* d) {
  if (!d || d->reserved[0] || d->reserved[1]) return SNN_ERR_INVALID_ARG;
  if (d->M < 0 || d->N < 1 || d->group < 0) return SNN_ERR_INVALID_ARG;
  if (d->dtype < SNN_F32 || d->dtype > SNN_F16 || d->res_dtype < SNN_F32 || d->res_dtype > SNN_F16)
    return SNN_ERR_INVALID_ARG;
  if (d->gate < SNN_GATE_NONE || d->gate > SNN_GATE_SILU) return SNN_ERR_INVALID_ARG;
  if (!(d->eps > 0.0f) || !std::isfinite(d->eps)) return SNN_ERR_INVALID_ARG;
  if (d->group && d->N % d->group) return SNN_ERR_INVALID_ARG;
  if (d->N > kMaxN || d->M > (int64_t(1) << 40)) return SNN_ERR_UNSUPPORTED;
  if (d->res_dtype != SNN_F32 && d->res_dtype != d->dtype) return SNN_ERR_UNSUPPORTED;
  if (d->group && d->group != d->N &&
      (d->group < 8 || d->group > 256 || (d->group & (d->group - 1))))
    return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

const void* data_of(const snn_rows* x) { return x ? x->data : nullptr; }

// A matrix that may be absent; *vec is cleared where its rows are not whole
// 16-byte vectors.
snn_status_t take(const snn_norm_desc* d, const snn_rows* x, int dtype, Rows* out, bool* vec) {
  *out = Rows{nullptr, 0};
  if (!data_of(x)) return SNN_OK;
  if (!aligned16(x->data)) return SNN_ERR_ALIGNMENT;
  if (d->M > 1 && (x->ld < d->N || x->ld > (int64_t(1) << 40))) return SNN_ERR_INVALID_ARG;
  if (d->M > 1 && x->ld % 8) *vec = false;
  *out = Rows{x->data, x->ld};
  return SNN_OK;
}

struct Launch {
  const Args& g;
  bool bwd;
  int64_t blocks;
  cudaStream_t st;
};

// Rows in shared memory: up to three, as many as fit beside the other blocks
// of an SM (and the sums of long rows).
template <typename K>
cudaError_t launch_staged(K* kernel, const Launch& l, int threads, int teams, int stage, size_t fixed,
                          int resident, int least_stages) {
  constexpr size_t kPerSm = 224 * 1024;
  Args g = l.g;
  g.stages = 3;
  while (g.stages > least_stages && g.stages * (size_t)teams * stage + fixed + 1024 > kPerSm / resident) --g.stages;
  size_t smem = g.stages * (size_t)teams * stage + fixed;
  // the teams' sums of short rows
  const size_t all = teams > 1 ? (size_t)teams * 2 * 32 * E * sizeof(float) : 0;
  if (smem < all) smem = all;
  // with the kernel's static shared memory, past the limit that needs no asking
  const size_t ask = smem + 1024 > 48 * 1024 && smem <= 48 * 1024 ? 48 * 1024 + 16 : smem;
  const cudaError_t e = ensure_smem((const void*)kernel, ask);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3((unsigned)l.blocks), dim3(threads), smem, l.st, g);
}

template <typename T, typename R, bool VEC, int TPR>
cudaError_t launch_tpr(const Launch& l) {
  constexpr int kThreads = kBlockThreads<TPR>;
  if (!l.bwd)
    return launch_staged(norm_fwd<T, R, VEC, TPR>, l, kThreads, kTeams<TPR>,
                         fwd_stage(l.g.N, sizeof(T), sizeof(R)), 0, 1024 / kThreads, 2);
  return launch_staged(norm_bwd<T, R, VEC, TPR>, l, kThreads, kTeams<TPR>,
                       VEC && TPR < 1024 ? 0 : bwd_stage(l.g.N, sizeof(T), sizeof(R)),
                       TPR == 1024 ? 2 * E * sizeof(float) * TPR : 0,
                       TPR == 1024 ? 1 : kBwdThreads / kThreads, 1);
}

template <typename T, typename R, bool VEC>
cudaError_t launch_vec(const Launch& l) {
  switch (row_threads(l.g.N)) {
    case 32: return launch_tpr<T, R, VEC, 32>(l);
    case 64: return launch_tpr<T, R, VEC, 64>(l);
    case 128: return launch_tpr<T, R, VEC, 128>(l);
    case 256: return launch_tpr<T, R, VEC, 256>(l);
    case 512: return launch_tpr<T, R, VEC, 512>(l);
    default: return launch_tpr<T, R, VEC, 1024>(l);
  }
}

template <typename T, typename R>
cudaError_t launch_types(const Launch& l, bool vec) {
  return vec ? launch_vec<T, R, true>(l) : launch_vec<T, R, false>(l);
}

cudaError_t launch(const snn_norm_desc* d, const Launch& l, bool vec) {
  if (d->dtype == SNN_F32) return launch_types<float, float>(l, vec);
  if (d->dtype == SNN_BF16)
    return d->res_dtype == SNN_F32 ? launch_types<__nv_bfloat16, float>(l, vec)
                                   : launch_types<__nv_bfloat16, __nv_bfloat16>(l, vec);
  return d->res_dtype == SNN_F32 ? launch_types<__half, float>(l, vec)
                                 : launch_types<__half, __half>(l, vec);
}

Args base_args(const snn_norm_desc* d, const float* w_post, const float* scale, const float* w_pre) {
  Args g = {};
  g.M = d->M;
  g.N = (int)d->N;
  g.group = d->group ? (int)d->group : g.N;
  g.gate = d->gate;
  g.eps = d->eps;
  g.w_post = w_post;
  g.scale = scale;
  g.w_pre = w_pre;
  return g;
}

// Rows move in vectors when N and every row stride are whole ones.
snn_status_t finish(const snn_norm_desc* d, bool* vec) {
  if (d->N % 8) *vec = false;
  if (!*vec && d->group && d->group != d->N) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}

}  // namespace norm
}  // namespace snn

using namespace snn::norm;

extern "C" {

size_t snn_norm_desc_size(void) { return sizeof(snn_norm_desc); }

size_t snn_block_norm_workspace_bytes(int64_t M, int64_t N) {
  if (M < 0 || N < 1 || N > kMaxN) return 0;
  const size_t b = (size_t)bwd_blocks(M, N) * 2 * (size_t)N * sizeof(float);
  return b < 256 ? 256 : b;
}

snn_status_t snn_block_norm_fwd(const snn_norm_desc* desc, const snn_rows* r, const snn_rows* a,
                                const snn_rows* z, const float* w_post, const float* res_scale,
                                const float* w_pre, const snn_rows* r_out, const snn_rows* y,
                                snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  if (desc->M == 0) return SNN_OK;
  const bool block = data_of(a) != nullptr;
  if (!data_of(r) || block != (data_of(r_out) != nullptr)) return SNN_ERR_INVALID_ARG;
  if ((w_pre != nullptr) != (data_of(y) != nullptr) || (!block && !w_pre)) return SNN_ERR_INVALID_ARG;
  if ((data_of(z) != nullptr) != (block && desc->gate != SNN_GATE_NONE)) return SNN_ERR_INVALID_ARG;
  const void* ptrs[3] = {w_post, res_scale, w_pre};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  Args g = base_args(desc, w_post, res_scale, w_pre);
  bool vec = true;
  const int io = desc->dtype, res = desc->res_dtype;
  if ((s = take(desc, r, res, &g.r, &vec)) != SNN_OK || (s = take(desc, a, io, &g.a, &vec)) != SNN_OK ||
      (s = take(desc, z, io, &g.z, &vec)) != SNN_OK || (s = take(desc, r_out, res, &g.ro, &vec)) != SNN_OK ||
      (s = take(desc, y, io, &g.y, &vec)) != SNN_OK || (s = finish(desc, &vec)) != SNN_OK)
    return s;
  const Launch l{g, false, blocks_for(desc->M, desc->N, 1024), reinterpret_cast<cudaStream_t>(stream)};
  return launch(desc, l, vec) == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

snn_status_t snn_block_norm_bwd(const snn_norm_desc* desc, const snn_rows* r_out,
                                const snn_rows* a, const snn_rows* z, const float* w_post,
                                const float* res_scale, const float* w_pre,
                                const snn_rows* grad_r_out, const snn_rows* grad_y,
                                const snn_rows* grad_r, const snn_rows* grad_a,
                                const snn_rows* grad_z, float* grad_w_post, float* grad_scale,
                                float* grad_w_pre, void* ws, size_t ws_bytes, snn_stream_t stream) {
  snn_status_t s = check_desc(desc);
  if (s != SNN_OK) return s;
  const bool block = data_of(a) != nullptr, pre = data_of(grad_y) != nullptr;
  const bool params = grad_w_post || grad_scale || grad_w_pre;
  if (desc->M > 0) {
    if (!pre && !data_of(grad_r_out)) return SNN_ERR_INVALID_ARG;
    if (pre && (!w_pre || !data_of(r_out))) return SNN_ERR_INVALID_ARG;
    if ((data_of(z) != nullptr) != (block && desc->gate != SNN_GATE_NONE)) return SNN_ERR_INVALID_ARG;
    if (!block && (data_of(grad_a) || grad_w_post || grad_scale)) return SNN_ERR_INVALID_ARG;
    if (!data_of(z) && data_of(grad_z)) return SNN_ERR_INVALID_ARG;
  }
  const void* ptrs[7] = {w_post, res_scale, w_pre, grad_w_post, grad_scale, grad_w_pre, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return SNN_ERR_ALIGNMENT;
  if (params && (!ws || ws_bytes < snn_block_norm_workspace_bytes(desc->M, desc->N)))
    return SNN_ERR_WORKSPACE;
  Args g = base_args(desc, w_post, res_scale, w_pre);
  bool vec = true;
  const int io = desc->dtype, res = desc->res_dtype;
  if ((s = take(desc, r_out, res, &g.ro, &vec)) != SNN_OK || (s = take(desc, a, io, &g.a, &vec)) != SNN_OK ||
      (s = take(desc, z, io, &g.z, &vec)) != SNN_OK ||
      (s = take(desc, grad_r_out, res, &g.gro, &vec)) != SNN_OK ||
      (s = take(desc, grad_y, io, &g.gy, &vec)) != SNN_OK || (s = take(desc, grad_r, res, &g.gr, &vec)) != SNN_OK ||
      (s = take(desc, grad_a, io, &g.ga, &vec)) != SNN_OK || (s = take(desc, grad_z, io, &g.gz, &vec)) != SNN_OK ||
      (s = finish(desc, &vec)) != SNN_OK)
    return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const int64_t blocks = bwd_blocks(desc->M, desc->N);
  cudaError_t e = cudaSuccess;
  if (desc->M > 0) {
    g.part = params ? static_cast<float*>(ws) : nullptr;
    const Launch l{g, true, blocks, st};
    e = launch(desc, l, vec);
  }
  if (e == cudaSuccess && params)
    e = snn::launch_pdl(norm_sum, dim3((unsigned)((2 * desc->N + 31) / 32)), dim3(1024), 0, st,
                        static_cast<const float*>(ws), (int)blocks, (int)desc->N, w_post,
                        res_scale, grad_w_post, grad_scale, grad_w_pre);
  return e == cudaSuccess ? SNN_OK : SNN_ERR_CUDA;
}

}  // extern "C"
