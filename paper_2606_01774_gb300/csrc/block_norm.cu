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
// Bound by bytes: every row is read once and written once.  A team of threads takes a row,
// eight elements next to each other per thread; a team is a warp for rows of up to 256 elements
// (eight teams to a CTA), a CTA for rows of up to 4096, a cluster of two or four CTAs for longer
// ones.  Teams walk their rows; a thread copies its own elements of the next rows to
// its own places in shared memory meanwhile (cp.async), so loads need no barrier, and
// only the sums over a row meet other threads.  The gradient of a weight is summed over a team's
// rows in registers, then over the CTA, and the CTAs' sums in a fixed order by a second kernel.
#include "async.cuh"
#include "common.cuh"
#include "kernels.h"
#include "pdl.cuh"
#include "piece.cuh"

namespace flare {

namespace {

constexpr int kMaxTeam = 512;                // threads of a CTA, eight elements each
constexpr int kBwdVectors = 2;               // of eight elements per thread, backward
constexpr int kMaxCols = 8 * kMaxTeam;       // columns of a CTA
constexpr int kMaxCluster = 4;

__device__ __forceinline__ float exp2f_fast(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Sums over a row, the same in every thread of it.  Calls alternate between two buffers, so that
// one is written again only after a barrier that follows its last reader.
struct RowSum {
  float (*buf)[2][16];           // [2][values][warps]
  float (*far)[2][kMaxCluster];  // [2][values][CTAs of the cluster]
  int cluster, rank, turn;

  // A warp's two sums go down one tree: its halves swap one value each, so that the lower
  // half holds the first and the upper half the second.
  template <int K>
  __device__ __forceinline__ void operator()(float (&v)[K]) {
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    const bool upper = K == 2 && lane >= 16;
    float x = v[0];
    if (K == 2) x = (upper ? v[K - 1] : v[0]) + __shfl_xor_sync(~0u, upper ? v[0] : v[K - 1], 16);
    else x += __shfl_xor_sync(~0u, x, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
    if (warps > 1) {  // a row of more than a warp
      turn ^= 1;
      if (K == 2 ? (lane & 15) == 0 : lane == 0) buf[turn][upper][threadIdx.x >> 5] = x;
      __syncthreads();
      x = (lane & 15) < warps ? buf[turn][upper][lane & 15] : 0.f;
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
    if (cluster == 1) return;
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

// 1 / (1 + e^-z).  The exponent z log2 e in two parts (its rounding would be a relative error
// of |z| 2^-24), the quotient by the fast reciprocal: 2^-22 in all.  Zero from z = -87.3 down,
// where the quotient leaves the normal numbers.
__device__ __forceinline__ float sigmoid(float z) {
  constexpr float kLog2e = 1.44269504089f, kRest = 1.92596300e-8f;
  const float t = z * -kLog2e, hi = t > 127.f ? 127.f : t;  // a NaN stays one
  const float lo = fmaf(z, -kLog2e, -hi) - z * kRest;
  const float e = exp2f_fast(hi);
  return __fdividef(1.f, 1.f + (fabsf(hi) < 127.f ? fmaf(e, lo * 0.693147181f, e) : e));
}

// Sigmoids of eight gates (nothing for a gate that is taken as it is).
__device__ __forceinline__ void sigmoid8(int kind, const uint64_t (&z)[4], uint64_t (&s)[4]) {
  if (kind == FLARE_ACT_NONE) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float z0, z1;
    f2_split(z[i], z0, z1);
    s[i] = f2(sigmoid(z0), sigmoid(z1));
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

// A thread's own places in shared memory: its eight elements of each input of a row.
template <typename T>
struct Slots {
  static constexpr int M = 8 / Piece<T>::N;
  uint4* at;   // of this thread, piece 0
  int pieces;  // from one piece to the next: threads of the CTA

  __device__ __forceinline__ void fetch(int array, const T* src) const {
#pragma unroll
    for (int i = 0; i < M; ++i)
      cp_async16(at + (array * M + i) * pieces, reinterpret_cast<const uint4*>(src) + i);
  }
  __device__ __forceinline__ void read(int array, uint64_t (&x)[4]) const {
    uint4 u[M];
#pragma unroll
    for (int i = 0; i < M; ++i) u[i] = at[(array * M + i) * pieces];
    load_pairs<T>(u, x);
  }
};

// A thread's own weights in shared memory: after the block (times alpha), before the next.
struct Weights {
  uint4* at;
  int pieces;

  __device__ __forceinline__ void fill(const BlockNormParams& p, int c) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float4 w = make_float4(1.f, 1.f, 1.f, 1.f);
      if (p.wpost) w = reinterpret_cast<const float4*>(p.wpost + (p.shared ? c % p.G : c))[i];
      w.x *= p.alpha, w.y *= p.alpha, w.z *= p.alpha, w.w *= p.alpha;
      reinterpret_cast<float4*>(at)[i * pieces] = w;
      w = make_float4(1.f, 1.f, 1.f, 1.f);
      if (p.wpre) w = reinterpret_cast<const float4*>(p.wpre + c)[i];
      reinterpret_cast<float4*>(at)[(2 + i) * pieces] = w;
    }
  }
  __device__ __forceinline__ void read(int kind, uint64_t (&x)[4]) const {
    const uint4 u[2] = {at[2 * kind * pieces], at[(2 * kind + 1) * pieces]};
    load_pairs<float>(u, x);
  }
};

__device__ __forceinline__ void wait_rows(int later) {
  if (later >= 3) cp_async_wait<3>();
  else if (later == 2) cp_async_wait<2>();
  else cp_async_wait<1>();
}

struct Shape {
  int team, teams, cluster, ctas;  // threads of a CTA's team, teams of a CTA, CTAs of a cluster
  int cols;                        // columns of a CTA
  int arrays, stages;              // forward: inputs, and rows in flight
  int smem;
};

}  // namespace

template <typename T, bool GATE>
__global__ void __launch_bounds__(kMaxTeam, 2)
    block_norm_kernel(const __grid_constant__ BlockNormParams p, const __grid_constant__ Shape s) {
  extern __shared__ __align__(16) char smem[];
  __shared__ float buf[2][2][16], far[2][2][kMaxCluster];
  const int thread = threadIdx.y * blockDim.x + threadIdx.x;
  const int threads = blockDim.x * blockDim.y;
  const int rank = blockIdx.x % s.cluster;
  RowSum row_sum{buf, far, s.cluster, rank, 0};
  const int c = rank * s.cols + threadIdx.x * 8;
  const bool mine = threadIdx.x * 8 < s.cols && c < p.W;
  const bool heads = p.post && p.G != p.W;
  const float per_group = 1.f / (float)p.G, per_row = 1.f / (float)p.W;
  const Weights weights{reinterpret_cast<uint4*>(smem) + thread, threads};
  uint4* ring = reinterpret_cast<uint4*>(smem) + 4 * threads + thread;
  const int stage = s.arrays * Slots<T>::M * threads;
  constexpr int kGate = 1, kRes = 1 + GATE;

  if (mine) weights.fill(p, c);
  if (s.cluster > 1) cluster_sync();  // every CTA runs before another writes to its memory
  const int64_t step = (int64_t)(gridDim.x / s.cluster) * blockDim.y;
  const int64_t first = (int64_t)(blockIdx.x / s.cluster) * blockDim.y + threadIdx.y;
  const auto fetch = [&](int64_t row, int at) {
    if (mine && row < p.T) {
      const Slots<T> to{ring + at * stage, threads};
      to.fetch(0, static_cast<const T*>(p.x) + row * p.x_stride + c);
      if (GATE) to.fetch(kGate, static_cast<const T*>(p.gate) + row * p.gate_stride + c);
      if (p.residual) to.fetch(kRes, static_cast<const T*>(p.residual) + row * p.W + c);
    }
    cp_async_commit();
  };
  for (int i = 0; i < s.stages - 1; ++i) fetch(first + i * step, i);
  int at = 0;
  for (int64_t row = first; row < p.T; row += step) {
    const int last = at == 0 ? s.stages - 1 : at - 1;
    fetch(row + (s.stages - 1) * step, last);
    wait_rows(s.stages - 1);
    const Slots<T> in{ring + at * stage, threads};
    at = at + 1 == s.stages ? 0 : at + 1;

    uint64_t y[4] = {}, t[4] = {}, w[4] = {};
    if (mine) {
      in.read(0, y);
      weights.read(0, w);
    }
    if (p.post) {
      float sum[1] = {dot8(y, y)};
      if (heads) sum[0] = lanes_sum(sum[0], p.G / 8);
      else row_sum(sum);
      const uint64_t q = f2_dup(rsqrtf(sum[0] * per_group + p.eps));
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = f2_mul(w[i], q);
    }
    if (GATE) {
      uint64_t sig[4] = {};
      if (mine) in.read(kGate, t);
      sigmoid8(p.act, t, sig);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = f2_mul(w[i], activation(p.act, t[i], sig[i]));
        t[i] = 0;
      }
    }
    if (p.residual && mine) in.read(kRes, t);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = f2_fma(y[i], w[i], t[i]);
    if (p.y && mine) store_pairs<T>(static_cast<T*>(p.y) + row * p.W + c, y);
    if (p.pre) {
      float squares[1] = {dot8(y, y)};
      row_sum(squares);
      const uint64_t r = f2_dup(rsqrtf(squares[0] * per_row + p.eps));
      if (mine) {
        weights.read(1, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = f2_mul(y[i], f2_mul(w[i], r));
        store_pairs<T>(static_cast<T*>(p.h) + row * p.W + c, y);
      }
    }
  }
  if (s.cluster > 1) cluster_sync();  // none leaves while another may write to its memory
}

// The shared memory of a backward thread, in 16-byte units: its weights, x of three rows, the other
// inputs of two.  Units lie THREADS apart, so that copies and reads of neighbouring threads
// meet neighbouring units, at distances known to the compiler.
template <typename T, bool GATE, bool PRE, int THREADS>
struct Own {
  static constexpr int V = kBwdVectors, M = Slots<T>::M;
  static constexpr int kGate = 0, kDy = GATE, kRes = kDy + 1, kDh = kDy + 2;
  static constexpr int kInputs = kDy + (PRE ? 3 : 1);
  static constexpr int kX = 4 * V, kRow = kX + 3 * V * M, kUnits = kRow + 2 * kInputs * V * M;
  static constexpr int kUnit = 16 * THREADS;  // bytes from unit to unit

  // after the block (kind 0), before the next (1)
  static __device__ __forceinline__ uint32_t weight(uint32_t own, int kind, int j) {
    return own + (kind * V + j) * 2 * kUnit;
  }
  static __device__ __forceinline__ uint32_t x(uint32_t own, int row, int j) {
    return own + (kX + (row * V + j) * M) * kUnit;
  }
  static __device__ __forceinline__ uint32_t input(uint32_t own, int row, int array, int j) {
    return own + (kRow + ((row * kInputs + array) * V + j) * M) * kUnit;
  }
  static __device__ __forceinline__ void fetch(uint32_t to, const T* src) {
#pragma unroll
    for (int i = 0; i < M; ++i)
      cp_async16(to + i * kUnit, reinterpret_cast<const uint4*>(src) + i);
  }
  template <typename U = T>
  static __device__ __forceinline__ void read(uint32_t at, uint64_t (&v)[4]) {
    constexpr int K = 8 / Piece<U>::N;
    uint4 u[K];
#pragma unroll
    for (int i = 0; i < K; ++i)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(u[i].x), "=r"(u[i].y), "=r"(u[i].z), "=r"(u[i].w)
                   : "r"(at + i * kUnit)
                   : "memory");
    load_pairs<U>(u, v);
  }
};

// Sixteen elements of a row per thread, in two vectors of eight.  The sum of the next row's squares
// goes along with this row's last sum, so x arrives a row ahead of the other inputs.  What a sum
// separates is read again after it, rather than held.  alpha enters by the rows' factors alone.
// What a call has, where the compiler knows it.
enum Form {
  kAny,
  kBlock,  // both norms over whole rows, a residual, and gradients at and of it: a block's end
  kOutput  // no norm before the next block: a layer's output stage
};

template <typename T, bool GATE, int FORM, int THREADS>
__global__ void __launch_bounds__(THREADS, 512 / THREADS)
    block_norm_bwd_kernel(const __grid_constant__ BlockNormParams p,
                          const __grid_constant__ Shape s) {
  constexpr bool FULL = FORM == kBlock;
  using O = Own<T, GATE, FORM != kOutput, THREADS>;
  constexpr int V = kBwdVectors;
  extern __shared__ __align__(16) char smem[];
  __shared__ float buf[2][2][16], far[2][2][kMaxCluster];
  const int thread = threadIdx.y * blockDim.x + threadIdx.x;
  const int threads = blockDim.x * blockDim.y;
  const int rank = blockIdx.x % s.cluster;
  RowSum row_sum{buf, far, s.cluster, rank, 0};
  const uint32_t own = (uint32_t)__cvta_generic_to_shared(smem) + thread * 16;
  // columns past the row's hold zeros throughout
  uint4* units = reinterpret_cast<uint4*>(smem) + thread;
#pragma unroll 1
  for (int i = 0; i < O::kUnits; ++i) units[i * THREADS] = make_uint4(0, 0, 0, 0);
  int c[V];
  bool mine[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int at = (j * blockDim.x + threadIdx.x) * 8;
    c[j] = rank * s.cols + at;
    mine[j] = at < s.cols && c[j] < p.W;
    if (!mine[j]) continue;
    for (int i = 0; i < 2; ++i) {
      float4* to = reinterpret_cast<float4*>(units + (2 * j + i) * THREADS);
      const float4 one = make_float4(1.f, 1.f, 1.f, 1.f);
      to[0] = p.wpost
                  ? reinterpret_cast<const float4*>(p.wpost + (p.shared ? c[j] % p.G : c[j]))[i]
                  : one;
      to[2 * V * THREADS] = p.wpre ? reinterpret_cast<const float4*>(p.wpre + c[j])[i] : one;
    }
  }
  const bool post_norm = FULL || p.post, pre_norm = FULL || (FORM == kAny && p.pre);
  const bool heads = !FULL && p.post && p.G != p.W;
  const float per_group = 1.f / (float)p.G, per_row = 1.f / (float)p.W;
  const bool use_res = FULL || (pre_norm && p.residual);  // y itself is needed by its norm alone
  if (s.cluster > 1) cluster_sync();
  const int64_t step = (int64_t)(gridDim.x / s.cluster) * blockDim.y;
  const int64_t first = (int64_t)(blockIdx.x / s.cluster) * blockDim.y + threadIdx.y;
  const auto fetch_x = [&](int64_t row, int at) {
    if (row >= p.T) return;
    const T* src = static_cast<const T*>(p.x) + row * p.x_stride;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (mine[j]) O::fetch(O::x(own, at, j), src + c[j]);
  };
  const auto fetch = [&](int64_t row, int at) {
    if (row >= p.T) return;
    const int64_t dense = row * p.W;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (!mine[j]) continue;
      const auto copy = [&](int array, const void* src, int64_t from) {
        O::fetch(O::input(own, at, array, j), static_cast<const T*>(src) + (from + c[j]));
      };
      if (GATE) copy(O::kGate, p.gate, row * p.gate_stride);
      if (use_res) copy(O::kRes, p.residual, dense);
      if (FULL || p.dy) copy(O::kDy, p.dy, dense);
      if (pre_norm) copy(O::kDh, p.dh, dense);
    }
  };
  uint64_t dwpost[V][4] = {}, dwpre[V][4] = {};

  fetch_x(first, 0);
  fetch(first, 0);
  fetch_x(first + step, 1);
  cp_async_commit();
  cp_async_wait<0>();
  const auto squares = [&](int at, int j) {  // of a vector, over its group where it has one
    uint64_t x[4];
    O::read(O::x(own, at, j), x);
    const float sum = dot8(x, x);
    return heads ? lanes_sum(sum, p.G / 8) : sum;
  };
  float q[V];
#pragma unroll
  for (int j = 0; j < V; ++j) q[j] = 1.f;
  if (post_norm) {
    float sum[1] = {0.f}, by[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[0] += by[j] = squares(0, j);
    if (!heads) row_sum(sum);
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = rsqrtf((heads ? by[j] : sum[0]) * per_group + p.eps);
  }
  int at = 0, x_at = 0;
  for (int64_t row = first; row < p.T; row += step) {
    const int x_next = x_at == 2 ? 0 : x_at + 1;
    fetch(row + step, at ^ 1);
    fetch_x(row + 2 * step, x_at == 0 ? 2 : x_at - 1);
    cp_async_commit();
    cp_async_wait<1>();  // this row, and the next one's x

    uint64_t g[V][4];
    if (pre_norm) {
      uint64_t y[V][4];
      float sums[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < V; ++j) {
        uint64_t x[4], w[4], t[4];
        O::read(O::input(own, at, O::kRes, j), y[j]);  // zeros where there is none
        O::read(O::x(own, x_at, j), x);
        O::template read<float>(O::weight(own, 0, j), w);
        if (GATE) {
          uint64_t sig[4];
          O::read(O::input(own, at, O::kGate, j), t);
          sigmoid8(p.act, t, sig);
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = f2_mul(w[i], activation(p.act, t[i], sig[i]));
        }
        const uint64_t qa = f2_dup(q[j] * p.alpha);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[j][i] = f2_fma(x[i], f2_mul(w[i], qa), y[j][i]);
        O::read(O::input(own, at, O::kDh, j), t);
        O::template read<float>(O::weight(own, 1, j), w);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = f2_mul(w[i], t[i]);
        sums[0] += dot8(y[j], y[j]);
        sums[1] += dot8(y[j], w);
      }
      row_sum(sums);
      const float r = rsqrtf(sums[0] * per_row + p.eps);
      const uint64_t rr = f2_dup(r), back = f2_dup(-(sums[1] * per_row * r * r * r));
#pragma unroll
      for (int j = 0; j < V; ++j) {
        uint64_t dh[4], w[4];
        O::read(O::input(own, at, O::kDh, j), dh);
        O::read(O::input(own, at, O::kDy, j), g[j]);
        O::template read<float>(O::weight(own, 1, j), w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint64_t d = f2_mul(dh[i], rr);
          dwpre[j][i] = f2_fma(d, y[j][i], dwpre[j][i]);
          g[j][i] = f2_fma(y[j][i], back, f2_fma(d, w[i], g[j][i]));
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) O::read(O::input(own, at, O::kDy, j), g[j]);
    }
    float sums[2] = {0.f, 0.f}, dot[V], next[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if ((FULL || p.dres) && mine[j]) store_pairs<T>(static_cast<T*>(p.dres) + (row * p.W + c[j]), g[j]);
      uint64_t x[4], w[4];
      O::read(O::x(own, x_at, j), x);
      O::template read<float>(O::weight(own, 0, j), w);
      const uint64_t qq = f2_dup(q[j]);
      if (GATE) {
        uint64_t z[4], sig[4];
        O::read(O::input(own, at, O::kGate, j), z);
        sigmoid8(p.act, z, sig);
        const uint64_t qa = f2_dup(q[j] * p.alpha);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint64_t n = f2_mul(x[i], f2_mul(w[i], qa));
          const uint64_t a = activation(p.act, z[i], sig[i]);
          z[i] = f2_mul(activation_slope(p.act, z[i], sig[i]), f2_mul(g[j][i], n));
          g[j][i] = f2_mul(g[j][i], a);
        }
        if (mine[j])
          store_pairs<T>(static_cast<T*>(p.dgate) + (row * p.gate_stride + c[j]), z);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dwpost[j][i] = f2_fma(g[j][i], f2_mul(x[i], qq), dwpost[j][i]);
        g[j][i] = f2_mul(g[j][i], w[i]);
      }
      if (post_norm) {
        dot[j] = dot8(x, g[j]);
        if (heads) dot[j] = lanes_sum(dot[j], p.G / 8);
        next[j] = row + step < p.T ? squares(x_next, j) : 0.f;
        sums[0] += dot[j];
        sums[1] += next[j];
      }
    }
    if (post_norm && !heads) row_sum(sums);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float qa = q[j] * p.alpha;
      if (post_norm) {
        const float inner = heads ? dot[j] : sums[0];
        const uint64_t back = f2_dup(-(inner * per_group * qa * q[j] * q[j]));
        uint64_t x[4];
        O::read(O::x(own, x_at, j), x);
#pragma unroll
        for (int i = 0; i < 4; ++i) g[j][i] = f2_fma(x[i], back, f2_mul(g[j][i], f2_dup(qa)));
        q[j] = rsqrtf((heads ? next[j] : sums[1]) * per_group + p.eps);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) g[j][i] = f2_mul(g[j][i], f2_dup(qa));
      }
      if (mine[j]) store_pairs<T>(static_cast<T*>(p.dx) + (row * p.x_stride + c[j]), g[j]);
    }
    at ^= 1;
    x_at = x_next;
  }
  if (s.cluster > 1) cluster_sync();
  pdl_launch_next();
  if (!p.part) return;
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) dwpost[j][i] = f2_mul(dwpost[j][i], f2_dup(p.alpha));

  // the CTA's sums: [CTAs][post columns], then [CTAs][W] before the next block
  const int wide = p.shared ? p.G : p.W;
  float* post = p.part + (int64_t)(p.shared ? blockIdx.x : blockIdx.x / s.cluster) * wide;
  float* pre = p.part + (int64_t)gridDim.x * wide + (int64_t)(blockIdx.x / s.cluster) * p.W;
  if (!p.shared && blockDim.y == 1) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (mine[j]) {
        store_pairs<float>(post + c[j], dwpost[j]);
        store_pairs<float>(pre + c[j], dwpre[j]);
      }
    }
    return;
  }
  float* sums = reinterpret_cast<float*>(smem);  // [teams][columns]
  const int cols = blockDim.x * 8 * V, from = rank * s.cols;
  const int used = min(min(cols, s.cols), p.W - from);
  for (int kind = 0; kind < 2; ++kind) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j)
      store_pairs<float>(sums + threadIdx.y * cols + (j * blockDim.x + threadIdx.x) * 8,
                         kind ? dwpre[j] : dwpost[j]);
    __syncthreads();
    const bool by_group = p.shared && !kind;
    const int n = by_group ? p.G : used;
    for (int i = thread; i < n; i += threads) {
      float total = 0.f;
      for (int team = 0; team < blockDim.y; ++team)
        for (int k = i; k < used; k += n) total += sums[team * cols + k];
      if (by_group) post[i] = total;
      else (kind ? pre : post)[from + i] = total;
    }
  }
}

// The CTAs' weight gradients joined: 32 columns a CTA, its warps one partial sum in 32 each,
// added in order at the end.
__global__ void __launch_bounds__(1024)
    block_norm_weights_kernel(const __grid_constant__ BlockNormParams p, int ctas, int cluster) {
  __shared__ float buf[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int wide_post = p.shared ? p.G : p.W;
  const bool post = blockIdx.y == 0;
  float* out = post ? p.dwpost : p.dwpre;
  const int wide = post ? wide_post : p.W, c = blockIdx.x * 32 + lane;
  pdl_wait();
  if (!out || blockIdx.x * 32 >= wide) return;
  const int n = post && p.shared ? ctas : ctas / cluster;
  float sum = 0.f;
  if (c < wide) {
    const float* at = p.part + (post ? 0 : (int64_t)ctas * wide_post) + c;
#pragma unroll 4
    for (int i = warp; i < n; i += 32) sum += at[(int64_t)i * wide];
  }
  buf[warp][lane] = sum;
  __syncthreads();
  sum = warp_sum(buf[lane][warp]);
  if (lane == 0 && blockIdx.x * 32 + warp < wide) out[blockIdx.x * 32 + warp] = sum;
}

namespace {

// The teams of a call on T rows of W elements.
Shape teams_for(int W, int vectors) {
  Shape s = {};
  s.cluster = W <= kMaxCols ? 1 : W <= 2 * kMaxCols ? 2 : 4;
  // whole groups of up to 256 columns to a CTA
  s.cols = s.cluster == 1 ? W : (W / s.cluster + 255) / 256 * 256;
  s.team = (s.cols + 256 * vectors - 1) / (256 * vectors) * 32;
  s.teams = s.team == 32 ? 8 / vectors : 1;
  return s;
}

// One CTA or cluster per row until every SM has as many as it holds.
void set_ctas(Shape& s, int T, int per_sm, int num_sms) {
  const int fit = (226 << 10) / (s.smem + 2048);
  per_sm = fit < 1 ? 1 : fit < per_sm ? fit : per_sm;
  const int rows = (T + s.teams - 1) / s.teams, clusters = per_sm * num_sms / s.cluster;
  s.ctas = (rows < clusters ? rows : clusters) * s.cluster;
}

Shape forward_shape(const BlockNormParams& p, bool bf16, int num_sms) {
  Shape s = teams_for(p.W, 1);
  const int threads = s.team * s.teams;
  const int per_sm = threads > 256 ? 2 : threads > 128 ? 4 : 8;
  s.arrays = 1 + (p.gate != nullptr) + (p.residual != nullptr);
  // weights, and as many rows as there is room for
  const int own = threads * 64, row = threads * (bf16 ? 16 : 32) * s.arrays;
  const int most = (220 << 10) / per_sm - 2048;
  s.stages = 2;
  while (s.stages < 4 && own + row * (s.stages + 1) <= most) ++s.stages;
  s.smem = own + row * s.stages;
  set_ctas(s, p.T, per_sm, num_sms);
  return s;
}

// Threads whose shared memory a backward CTA has room for.
int backward_threads(const Shape& s) { return s.team * s.teams <= 128 ? 128 : 256; }

template <typename T, bool GATE, bool PRE>
constexpr int units_of() {
  return Own<T, GATE, PRE, 1>::kUnits;
}

Shape backward_shape(int T, int W, bool gate, bool pre, bool bf16, int num_sms) {
  using B = __nv_bfloat16;
  Shape s = teams_for(W, kBwdVectors);
  const int units = bf16 ? pre ? gate ? units_of<B, true, true>() : units_of<B, false, true>()
                               : gate ? units_of<B, true, false>() : units_of<B, false, false>()
                         : pre ? gate ? units_of<float, true, true>() : units_of<float, false, true>()
                               : gate ? units_of<float, true, false>()
                                      : units_of<float, false, false>();
  s.smem = backward_threads(s) * 16 * units;
  set_ctas(s, T, 512 / backward_threads(s), num_sms);
  return s;
}

cudaError_t run(void (*kernel)(BlockNormParams, Shape), const BlockNormParams& p, const Shape& s,
                cudaStream_t stream) {
  cudaError_t e =
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, s.smem);
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

template <typename T>
cudaError_t run_forward(const BlockNormParams& p, const Shape& s, cudaStream_t stream) {
  return run(p.gate ? block_norm_kernel<T, true> : block_norm_kernel<T, false>, p, s, stream);
}

template <typename T, bool GATE, int FORM>
cudaError_t run_backward(const BlockNormParams& p, const Shape& s, cudaStream_t stream) {
  return run(backward_threads(s) == 128 ? block_norm_bwd_kernel<T, GATE, FORM, 128>
                                        : block_norm_bwd_kernel<T, GATE, FORM, 256>,
             p, s, stream);
}

template <typename T, bool GATE>
cudaError_t run_backward(const BlockNormParams& p, const Shape& s, cudaStream_t stream) {
  if (!p.pre) return run_backward<T, GATE, kOutput>(p, s, stream);
  if (p.post && p.G == p.W && p.residual && p.dy && p.dres)
    return run_backward<T, GATE, kBlock>(p, s, stream);
  return run_backward<T, GATE, kAny>(p, s, stream);
}

template <typename T>
cudaError_t run_backward(const BlockNormParams& p, const Shape& s, cudaStream_t stream) {
  return p.gate ? run_backward<T, true>(p, s, stream) : run_backward<T, false>(p, s, stream);
}

}  // namespace

cudaError_t launch_block_norm(const BlockNormParams& p, bool bf16, int num_sms,
                              cudaStream_t stream) {
  if (p.T == 0) return cudaSuccess;
  const Shape s = forward_shape(p, bf16, num_sms);
  note_launches(1);
  return bf16 ? run_forward<__nv_bfloat16>(p, s, stream) : run_forward<float>(p, s, stream);
}

int block_norm_bwd_ctas(int T, int W, bool pre, bool bf16, int num_sms) {
  // a gate only makes it fewer
  return T ? backward_shape(T, W, false, pre, bf16, num_sms).ctas : 0;
}

cudaError_t launch_block_norm_bwd(const BlockNormParams& p, bool bf16, int num_sms,
                                  cudaStream_t stream) {
  const bool weights = p.dwpost || p.dwpre;
  if (p.T == 0 && !weights) return cudaSuccess;
  Shape s = {};
  s.cluster = 1;
  if (p.T > 0) {
    s = backward_shape(p.T, p.W, p.gate != nullptr, p.pre, bf16, num_sms);
    note_launches(1);
    const cudaError_t e =
        bf16 ? run_backward<__nv_bfloat16>(p, s, stream) : run_backward<float>(p, s, stream);
    if (e != cudaSuccess) return e;
  }
  if (weights) {  // of no rows: zeros
    note_launches(1);
    return pdl_launch(block_norm_weights_kernel, dim3((unsigned)(p.W + 31) / 32, 2), 1024, 0,
                      stream, p.T > 0, 1, p, s.ctas, s.cluster);
  }
  return cudaSuccess;
}

}  // namespace flare
