// Rows of the norms: a row's values in registers and shared memory, its sums, and
// the plan of threads and blocks (block_norm.cu, layer_norm.cu).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

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
template <int TPR, int MOST = 3>
struct RowSum {
  float (*scratch)[MOST][32];  // [2][value][warp]
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

// Host side

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

// Threads of a row, eight channels each.
inline int row_threads(int64_t N) {
  return N <= 256 ? 32 : N <= 512 ? 64 : N <= 1024 ? 128 : N <= 2048 ? 256 : N <= 4096 ? 512 : 1024;
}

// Blocks for M rows with `threads` of them on an SM; from the shape alone, so
// that a shape always sums in the same order.
inline int64_t blocks_for(int64_t M, int64_t N, int threads) {
  const int tpr = row_threads(N), block = tpr == 32 ? 256 : tpr;
  const int64_t resident = (int64_t)kSms * (threads > block ? threads / block : 1);
  return least(resident, tpr == 32 ? (M + 7) / 8 : M);
}
inline int64_t bwd_blocks(int64_t M, int64_t N) { return blocks_for(M, N, kBwdThreads); }

inline const void* data_of(const snn_rows* x) { return x ? x->data : nullptr; }

}  // namespace norm
}  // namespace snn
