// The norm, gate and scaled residual after a block and the norm before the next one,
// and their gradients.
//
//   n = x q w,  q = rsqrt(mean_G x^2 + eps)      u = n act(gate)
//   y = residual + alpha u                       h = y r w', r = rsqrt(mean y^2 + eps)
//
//   m = w' dh            g = dy + r (m - y r^2 mean(y m))         dw' = sum_rows dh y r
//   du = alpha g         dgate = du n act'(gate)                  dresidual = g
//   dn = du act(gate)    dx = q (w dn - x q^2 mean_G(x w dn))     dw = sum_rows dn x q
//
// Bound by bytes: every row is read once and written once.  A team of warps takes a row, eight or
// sixteen elements per thread; several teams share a CTA, rows that one CTA cannot hold take a
// cluster of two or four.  Teams walk their rows; a thread copies its own elements
// of the next rows to its own places in shared memory meanwhile (cp.async), so loads need no
// barrier, and only the sums over a row meet other threads.  16384 bf16 rows of 4096 with both
// norms and a residual: forward 89 us (6.0 TB/s, a copy's rate being 6.8), backward 132 us
// (6.1 TB/s).  Where rows are so wide or inputs so many that two rows of all of them fill an SM's
// shared memory, loads wait for sums: 8960 gated bf16 rows of 6400 with norms per head backward
// 286 us (3.2 TB/s).
#pragma once

#include <cuda_runtime.h>

#include "async.cuh"
#include "common.cuh"
#include "kernels.h"
#include "piece.cuh"

namespace flare {

namespace {  // each source file its own kernels

constexpr int kMaxWarps = 32;  // of a CTA
constexpr int kMaxCluster = 4;
constexpr int kSmem = 228 << 10, kSmemMost = 227 << 10;  // of an SM, and of a CTA
constexpr int kSmemStatic = 2 * 2 * (kMaxWarps + kMaxCluster) * 4;  // RowSum's
constexpr int kSmemOwn = kSmemStatic + 1024;  // besides the rows', with what the system keeps

__device__ __forceinline__ float exp2f_fast(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Sums over a row, the same in every thread of its team.  Calls alternate between two buffers, so
// that one is written again only after a barrier that follows its last reader.  SIMPLE: one team
// of 2 to 16 warps in the CTA, and no cluster.
template <bool SIMPLE>
struct RowSum {
  float (*buf)[2][kMaxWarps];    // [2][values][warps of the CTA]
  float (*far)[2][kMaxCluster];  // [2][values][CTAs of the cluster]
  int cluster, rank, turn;

  // A warp's two sums go down one tree: its halves swap one value each, so that the lower
  // half holds the first and the upper half the second.
  template <int K>
  __device__ __forceinline__ void operator()(float (&v)[K]) {
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    const int warp0 = SIMPLE ? 0 : threadIdx.y * warps;
    const bool upper = K == 2 && lane >= 16;
    float x = v[0];
    if (K == 2) x = (upper ? v[K - 1] : v[0]) + __shfl_xor_sync(~0u, upper ? v[0] : v[K - 1], 16);
    else x += __shfl_xor_sync(~0u, x, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
    if (SIMPLE || warps > 1) {  // a row of more than a warp
      turn ^= 1;
      if ((K == 2 ? lane & 15 : lane) == 0) buf[turn][upper][warp0 + (threadIdx.x >> 5)] = x;
      if constexpr (SIMPLE)
        __syncthreads();
      else
        asm volatile("bar.sync %0, %1;" ::"r"(1 + threadIdx.y), "r"(blockDim.x) : "memory");
      x = (lane & 15) < warps ? buf[turn][upper][warp0 + (lane & 15)] : 0.f;
      if (!SIMPLE && warps > 16 && (lane & 15) + 16 < warps) x += buf[turn][upper][(lane & 15) + 16];
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
    }
    if (K == 2) {
      const float other = __shfl_xor_sync(~0u, x, 16);
      v[0] = upper ? other : x;
      v[K - 1] = upper ? x : other;
    } else {
      v[0] = x;
    }
    if (SIMPLE || cluster == 1) return;
    if (threadIdx.x < cluster) {  // to every CTA of the cluster
#pragma unroll
      for (int k = 0; k < K; ++k) {
        uint32_t at;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                     : "=r"(at)
                     : "r"((uint32_t)__cvta_generic_to_shared(&far[turn][k][rank])),
                       "r"(threadIdx.x));
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v[k]) : "memory");
      }
    }
    __syncwarp();
    cluster_sync();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = 0.f;
      for (int i = 0; i < cluster; ++i) v[k] += far[turn][k][i];
    }
  }
};

// Sum over `lanes` neighbouring lanes.
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// 1 / (1 + e^-z) by the fast exponential and reciprocal.  For fp32 the exponent z log2 e is taken
// in two parts (its rounding is a relative error of |z| 2^-24): 2^-22 in all.  A NaN stays one; below
// -87.3, where the sigmoid is less than 2^-126, it is 0.
template <typename T>
__device__ __forceinline__ float sigmoid(float z) {
  constexpr float kLog2e = 1.44269504089f;
  if constexpr (sizeof(T) == 2) {
    return __fdividef(1.f, 1.f + exp2f_fast(z * -kLog2e));
  } else {
    constexpr float kRest = 1.92596300e-8f;  // log2 e - kLog2e
    // infinities would make the second part a NaN; the sigmoid of 126 is one, of -126 zero
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(z) : "f"(126.f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(z) : "f"(-126.f));
    const float hi = z * -kLog2e, lo = fmaf(z, -kLog2e, -hi) - z * kRest;
    return __fdividef(1.f, fmaf(exp2f_fast(hi), fmaf(lo, 0.693147181f, 1.f), 1.f));
  }
}

// Sigmoids of eight gates (nothing for a gate that is taken as it is).
template <typename T>
__device__ __forceinline__ void sigmoid8(int kind, const uint64_t (&z)[4], uint64_t (&s)[4]) {
  if (kind == FLARE_ACT_NONE) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float z0, z1;
    f2_split(z[i], z0, z1);
    s[i] = f2(sigmoid<T>(z0), sigmoid<T>(z1));
  }
}

// The gate's activation from the gate and its sigmoid.
__device__ __forceinline__ uint64_t activation(int kind, uint64_t z, uint64_t s) {
  return kind == FLARE_ACT_NONE ? z : kind == FLARE_ACT_SIGMOID ? s : f2_mul(z, s);
}

// Its derivative: 1, s (1 - s) or s (1 + z (1 - s)).
__device__ __forceinline__ uint64_t activation_slope(int kind, uint64_t z, uint64_t s) {
  const uint64_t one = f2_dup(1.f);
  if (kind == FLARE_ACT_NONE) return one;
  const uint64_t rest = f2_fma(s, f2_dup(-1.f), one);
  return f2_mul(s, kind == FLARE_ACT_SIGMOID ? rest : f2_fma(z, rest, one));
}

__device__ __forceinline__ float pair_sum(uint64_t v) {
  float a, b;
  f2_split(v, a, b);
  return a + b;
}

// sum of a_i b_i
__device__ __forceinline__ float dot8(const uint64_t (&a)[4], const uint64_t (&b)[4]) {
  uint64_t s = f2_mul(a[0], b[0]), t = f2_mul(a[1], b[1]);
  s = f2_fma(a[2], b[2], s);
  t = f2_fma(a[3], b[3], t);
  return pair_sum(f2_add(s, t));
}

// Where a thread's eight elements of a row lie.  In bf16 next to each other, sixteen bytes; in fp32
// half of them, and the other half 128 elements on, so that a warp's accesses are whole
// lines.  A warp has 256 elements either way.
template <typename T>
constexpr int kHalves = sizeof(T) == 4 ? 2 : 1;
constexpr int kFar = 128;

template <typename T>
__device__ __forceinline__ int first_column(int vector) {
  const int warp = (vector * blockDim.x + threadIdx.x) & ~31, lane = threadIdx.x & 31;
  return warp * 8 + lane * (8 / kHalves<T>);
}

// Four weights of the eight: the i-th column they start at.
template <typename T>
__device__ __forceinline__ int weight_column(int i) {
  return i * (kHalves<T> == 1 ? 4 : kFar);
}

template <typename T>
__device__ __forceinline__ void store_row(T* p, const uint64_t (&x)[4],
                                          const bool (&mine)[kHalves<T>]) {
  if constexpr (kHalves<T> == 1) {
    if (mine[0]) store_pairs<T>(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float f[4];
      f2_split(x[2 * i], f[0], f[1]);
      f2_split(x[2 * i + 1], f[2], f[3]);
      if (mine[i]) *reinterpret_cast<uint4*>(p + i * kFar) = Piece<float>::store(f);
    }
  }
}

// Sums of a_i b_i over the groups of the first four elements and of the other four.
template <typename T>
__device__ __forceinline__ void group_sums(const uint64_t (&a)[4], const uint64_t (&b)[4], int G,
                                           float (&s)[2]) {
  s[0] = pair_sum(f2_fma(a[1], b[1], f2_mul(a[0], b[0])));
  s[1] = pair_sum(f2_fma(a[3], b[3], f2_mul(a[2], b[2])));
  if (kHalves<T> == 1) {
    s[0] = s[1] = lanes_sum(s[0] + s[1], G / 8);
  } else if (G == 2 * kFar) {
    s[0] = s[1] = lanes_sum(s[0] + s[1], 32);
  } else {
    s[0] = lanes_sum(s[0], G / 4);
    s[1] = lanes_sum(s[1], G / 4);
  }
}

// The teams of a call.
struct Shape {
  int team, teams, cluster, ctas;  // threads of a CTA's team, teams of a CTA, CTAs of a cluster
  int cols;                        // columns of a CTA
  int arrays, stages;              // forward: inputs, and rows in flight
  int kind;                        // backward: which of the kernels
  int smem;

  bool simple() const { return teams == 1 && cluster == 1 && team > 32 && team <= 512; }
};

// On T rows of W elements, `vectors` of eight a thread, CTAs of up to `threads`; no team (cluster
// 0) where a row does not fit in a cluster.
inline Shape teams_for(int T, int W, int vectors, int threads, int num_sms) {
  Shape s = {};
  const int most = 8 * vectors * threads;
  s.cluster = W <= most ? 1 : W <= 2 * most ? 2 : W <= 4 * most ? 4 : 0;
  if (!s.cluster) return s;
  // whole groups of up to 256 columns to a CTA
  s.cols = s.cluster == 1 ? W : (W / s.cluster + 255) / 256 * 256;
  s.team = (s.cols + 256 * vectors - 1) / (256 * vectors) * 32;
  s.teams = s.cluster == 1 ? threads / s.team : 1;
  while (s.teams > 1 && T <= (s.teams - 1) * num_sms) --s.teams;  // every SM its rows first
  return s;
}

// One CTA or cluster for every `teams` rows, until the SMs have `per_sm` CTAs each.
inline void set_ctas(Shape& s, int T, int per_sm, int num_sms) {
  const int rows = T / s.teams + (T % s.teams != 0);  // T may be the last int
  const int clusters = per_sm * num_sms / s.cluster;
  s.ctas = (rows < clusters ? rows : clusters) * s.cluster;
}

inline cudaError_t launch_shape(void (*kernel)(BlockNormParams, Shape), const BlockNormParams& p,
                                const Shape& s, cudaStream_t stream) {
  // always the same limit: another thread's call may come between this one and the launch
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       kSmemMost - kSmemStatic);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)s.ctas);
  cfg.blockDim = dim3((unsigned)s.team, (unsigned)s.teams);
  cfg.dynamicSmemBytes = (size_t)s.smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)s.cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = s.cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, p, s);
}

}  // namespace

}  // namespace flare
