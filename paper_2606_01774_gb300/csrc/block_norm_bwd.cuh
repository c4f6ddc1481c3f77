// The backward kernel of block norms (block_norm.cuh has the formulas).
//
// The gradient of a weight is summed over a team's rows in registers, then over the CTA, and
// the CTAs' sums in a fixed order by a second kernel (block_norm.cu).
#pragma once

#include "block_norm.cuh"
#include "pdl.cuh"

namespace flare {

namespace {

// The shared memory of a backward thread, in 16-byte units: its weights, x and
// the other inputs of two rows.  Units lie THREADS apart, so that copies and reads of neighbouring threads
// meet neighbouring units, at distances known to the compiler.
template <typename T, bool GATE, bool PRE, int V, int THREADS>
struct Own {
  static constexpr int M = 8 / Piece<T>::N;  // units of eight elements
  static constexpr int kGate = 0, kDy = GATE, kRes = kDy + 1, kDh = kDy + 2;
  static constexpr int kInputs = kDy + (PRE ? 3 : 1);
  static constexpr int kX = 4 * V, kRow = kX + 2 * V * M, kUnits = kRow + 2 * kInputs * V * M;
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
  static __device__ __forceinline__ void fetch(uint32_t to, const T* src, const bool (&mine)[M]) {
#pragma unroll
    for (int i = 0; i < M; ++i)
      if (mine[i]) cp_async16(to + i * kUnit, src + i * kFar);
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

// A weight's gradients of a thread's elements of type T.
template <typename T>
__device__ __forceinline__ void store_weights(float* p, const uint64_t (&x)[4],
                                              const bool (&mine)[kHalves<T>]) {
  if constexpr (kHalves<T> == 1) {
    if (mine[0]) store_pairs<float>(p, x);
  } else {
    store_row<float>(p, x, mine);
  }
}

// What a call has, where the compiler knows it.
enum Form {
  kAny,
  kBlock,  // both norms over whole rows, a residual, and gradients at and of it: a block's end
  kOutput  // no norm before the next block: a layer's output stage
};

// V vectors of eight elements of a row per thread.  The sum of the next row's squares
// goes along with this row's last sum, so x arrives a row ahead of the other inputs.  What a sum
// separates is read again after it, rather than held: of 128 registers a thread the weights'
// gradients take 32.  alpha enters by the rows' factors alone.  With the form known 16384 rows of
// 4096 take 132 us, 150 without; 16384 bf16 rows of 16 heads, an output stage, 90 and 99 on CTAs of one
// kind.  Forms with a gate, but for the output stage's, pass 4 to 196 bytes a thread through local
// memory, kAny in fp32 24 without one.
template <typename T, bool GATE, int FORM, bool SIMPLE, int V, int THREADS>
__global__ void __launch_bounds__(THREADS, 512 / THREADS)
    block_norm_bwd_kernel(const __grid_constant__ BlockNormParams p,
                          const __grid_constant__ Shape s) {
  constexpr bool FULL = FORM == kBlock;
  using O = Own<T, GATE, FORM != kOutput, V, THREADS>;
  extern __shared__ __align__(16) char smem[];
  __shared__ float buf[2][2][kMaxWarps], far[2][2][kMaxCluster];
  const int thread = threadIdx.y * blockDim.x + threadIdx.x;
  const int threads = blockDim.x * blockDim.y;
  const int rank = blockIdx.x % s.cluster;
  RowSum<SIMPLE> row_sum{buf, far, s.cluster, rank, 0};
  const uint32_t own = (uint32_t)__cvta_generic_to_shared(smem) + thread * 16;
  uint4* units = reinterpret_cast<uint4*>(smem) + thread;
  constexpr int H = kHalves<T>;
  int c[V];
  bool mine[V][H];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int at = first_column<T>(j);
    c[j] = rank * s.cols + at;
#pragma unroll
    for (int i = 0; i < H; ++i)
      mine[j][i] = at + i * kFar < s.cols && c[j] + i * kFar < p.W;
  }
  // columns past the row's and inputs that the call has not hold zeros throughout
  if (!FULL || !mine[V - 1][H - 1]) {
#pragma unroll 1
    for (int i = 0; i < O::kUnits; ++i) units[i * THREADS] = make_uint4(0, 0, 0, 0);
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
    for (int j = 0; j < V; ++j) O::fetch(O::x(own, at, j), src + c[j], mine[j]);
  };
  const auto fetch = [&](int64_t row, int at) {
    if (row >= p.T) return;
    const int64_t dense = row * p.W;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const auto copy = [&](int array, const void* src, int64_t from) {
        O::fetch(O::input(own, at, array, j), static_cast<const T*>(src) + (from + c[j]), mine[j]);
      };
      if (GATE) copy(O::kGate, p.gate, row * p.gate_stride);
      if (use_res) copy(O::kRes, p.residual, dense);
      if (FULL || p.dy) copy(O::kDy, p.dy, dense);
      if (pre_norm) copy(O::kDh, p.dh, dense);
    }
  };
  uint64_t dwpost[V][4] = {}, dwpre[V][4] = {};

  fetch_x(first, 0);
  cp_async_commit();
  fetch(first, 0);
  cp_async_commit();
  fetch_x(first + step, 1);
  cp_async_commit();
  // the weights, all asked for before the first is put down, behind the first rows
  float4 w_post[V][2], w_pre[V][2];
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w_post[j][i] = w_pre[j][i] = make_float4(1.f, 1.f, 1.f, 1.f);
      if (!mine[j][i % H]) continue;
      const int at_w = c[j] + weight_column<T>(i);
      if (p.wpost)
        w_post[j][i] =
            *reinterpret_cast<const float4*>(p.wpost + (p.shared ? at_w % p.G : at_w));
      if (p.wpre) w_pre[j][i] = *reinterpret_cast<const float4*>(p.wpre + at_w);
    }
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (!mine[j][i % H]) continue;
      float4* to = reinterpret_cast<float4*>(units + (2 * j + i) * THREADS);
      to[0] = w_post[j][i];
      to[2 * V * THREADS] = w_pre[j][i];
    }
  cp_async_wait<2>();
  // of a vector, over its groups where it has some (else all of it in the first)
  const auto sums_of = [&](const uint64_t (&a)[4], const uint64_t (&b)[4], float (&sum)[2]) {
    if (heads) group_sums<T>(a, b, p.G, sum);
    else sum[0] = sum[1] = dot8(a, b);
  };
  const auto squares = [&](int at, int j, float (&sum)[2]) {
    uint64_t x[4];
    O::read(O::x(own, at, j), x);
    sums_of(x, x, sum);
  };
  float q[V][2];  // of a vector's halves
#pragma unroll
  for (int j = 0; j < V; ++j) q[j][0] = q[j][1] = 1.f;
  if (post_norm) {
    float sum[1] = {0.f}, by[V][2];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      squares(0, j, by[j]);
      sum[0] += by[j][0];
    }
    if (!heads) row_sum(sum);
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        q[j][i] = rsqrtf((heads ? by[j][i] : sum[0]) * per_group + p.eps);
  }
  int at = 0;
  for (int64_t row = first; row < p.T; row += step) {
    fetch(row + step, at ^ 1);
    cp_async_commit();
    cp_async_wait<2>();  // all but the next row: of this one the other inputs

    uint64_t g[V][4];
    if (pre_norm) {
      uint64_t y[V][4];
      float sums[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < V; ++j) {
        uint64_t x[4], w[4], t[4];
        O::read(O::input(own, at, O::kRes, j), y[j]);  // zeros where there is none
        O::read(O::x(own, at, j), x);
        O::template read<float>(O::weight(own, 0, j), w);
        if (GATE) {
          uint64_t sig[4];
          O::read(O::input(own, at, O::kGate, j), t);
          sigmoid8<T>(p.act, t, sig);
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = f2_mul(w[i], activation(p.act, t[i], sig[i]));
        }
        const uint64_t qa[2] = {f2_dup(q[j][0] * p.alpha), f2_dup(q[j][1] * p.alpha)};
#pragma unroll
        for (int i = 0; i < 4; ++i) y[j][i] = f2_fma(x[i], f2_mul(w[i], qa[i / 2]), y[j][i]);
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
    cp_async_wait<1>();  // the next row's x
    float sums[2] = {0.f, 0.f}, dot[V][2], next[V][2];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (FULL || p.dres)
        store_row<T>(static_cast<T*>(p.dres) + (row * p.W + c[j]), g[j], mine[j]);
      uint64_t x[4], w[4];
      O::read(O::x(own, at, j), x);
      O::template read<float>(O::weight(own, 0, j), w);
      const uint64_t qq[2] = {f2_dup(q[j][0]), f2_dup(q[j][1])};
      if (GATE) {
        uint64_t z[4], sig[4];
        O::read(O::input(own, at, O::kGate, j), z);
        sigmoid8<T>(p.act, z, sig);
        const uint64_t qa[2] = {f2_dup(q[j][0] * p.alpha), f2_dup(q[j][1] * p.alpha)};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint64_t n = f2_mul(x[i], f2_mul(w[i], qa[i / 2]));
          const uint64_t a = activation(p.act, z[i], sig[i]);
          z[i] = f2_mul(activation_slope(p.act, z[i], sig[i]), f2_mul(g[j][i], n));
          g[j][i] = f2_mul(g[j][i], a);
        }
        store_row<T>(static_cast<T*>(p.dgate) + (row * p.gate_stride + c[j]), z, mine[j]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dwpost[j][i] = f2_fma(g[j][i], f2_mul(x[i], qq[i / 2]), dwpost[j][i]);
        g[j][i] = f2_mul(g[j][i], w[i]);
      }
      if (post_norm) {
        sums_of(x, g[j], dot[j]);
        next[j][0] = next[j][1] = 0.f;
        if (row + step < p.T) squares(at ^ 1, j, next[j]);
        sums[0] += dot[j][0];
        sums[1] += next[j][0];
      }
    }
    if (post_norm && !heads) row_sum(sums);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      uint64_t x[4];
      if (post_norm) O::read(O::x(own, at, j), x);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float qa = q[j][k] * p.alpha;
        if (post_norm) {
          const float inner = heads ? dot[j][k] : sums[0];
          const uint64_t back = f2_dup(-(inner * per_group * qa * q[j][k] * q[j][k]));
#pragma unroll
          for (int i = 2 * k; i < 2 * k + 2; ++i)
            g[j][i] = f2_fma(x[i], back, f2_mul(g[j][i], f2_dup(qa)));
          q[j][k] = rsqrtf((heads ? next[j][k] : sums[1]) * per_group + p.eps);
        } else {
#pragma unroll
          for (int i = 2 * k; i < 2 * k + 2; ++i) g[j][i] = f2_mul(g[j][i], f2_dup(qa));
        }
      }
      store_row<T>(static_cast<T*>(p.dx) + (row * p.x_stride + c[j]), g[j], mine[j]);
    }
    fetch_x(row + 2 * step, at);
    cp_async_commit();
    at ^= 1;
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
      store_weights<T>(post + c[j], dwpost[j], mine[j]);
      store_weights<T>(pre + c[j], dwpre[j], mine[j]);
    }
    return;
  }
  bool all[H];
#pragma unroll
  for (int i = 0; i < H; ++i) all[i] = true;
  float* sums = reinterpret_cast<float*>(smem);  // [teams][columns]
  const int cols = blockDim.x * 8 * V, from = rank * s.cols;
  const int used = min(min(cols, s.cols), p.W - from);
  for (int kind = 0; kind < 2; ++kind) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j)
      store_weights<T>(sums + threadIdx.y * cols + first_column<T>(j), kind ? dwpre[j] : dwpost[j],
                       all);
    __syncthreads();
    // over the groups, of which every CTA of a cluster has whole ones: `from` is a multiple of G
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

// Vectors per thread and threads per CTA: what holds most of the rows in flight on an SM, and most
// warps.  (Rows of 4096 in bf16: two CTAs of 256 threads, 16 elements each; where inputs are so
// many or so wide that one CTA fills the shared memory, 512 threads.  Output stages would do better with
// fewer CTAs than it finds: 1021 fp32 rows of 16 heads 19.5 us, 16.3 by the kind that a call with a
// norm before the next block gets.)  Fewer rows may take another
// kind, with more CTAs: most_ctas, if given, becomes what any number of rows up to T_rows takes at most.
template <typename T, bool GATE, bool PRE>
Shape backward_shape(int T_rows, int W, int num_sms, int* most_ctas = nullptr) {
  Shape best = {};
  int best_score = 0;
  const auto consider = [&](int kind, int units, int vectors, int threads) {
    Shape s = teams_for(T_rows, W, vectors, threads, num_sms);
    s.smem = threads * 16 * units;
    if (!s.cluster || s.smem + kSmemStatic > kSmemMost) return;
    const int room = kSmem / (s.smem + kSmemOwn);
    const int per_sm = room < 512 / threads ? room : 512 / threads;
    if (most_ctas) {  // of this kind: a row to every CTA or cluster
      Shape one = s;
      one.teams = 1;
      set_ctas(one, T_rows, per_sm, num_sms);
      if (one.ctas > *most_ctas) *most_ctas = one.ctas;
    }
    const int used = per_sm * s.team * s.teams, warps = used / 32;
    // a cluster's barriers cost as much as half of the rows in flight, sixteen vectors as a warp
    const int score = used * vectors / (s.cluster > 1 ? 2 : 1) + 16 * warps;
    if (score <= best_score) return;
    best = s;
    best.kind = kind;
    set_ctas(best, T_rows, per_sm, num_sms);
    best_score = score;
  };
  consider(0, Own<T, GATE, PRE, 2, 1>::kUnits, 2, 128);
  consider(1, Own<T, GATE, PRE, 2, 1>::kUnits, 2, 256);
  consider(2, Own<T, GATE, PRE, 1, 1>::kUnits, 1, 512);
  if (sizeof(T) == 2) consider(3, Own<T, GATE, PRE, 2, 1>::kUnits, 2, 512);
  return best;
}

template <typename T, bool GATE, int FORM, bool SIMPLE>
cudaError_t run_backward(const BlockNormParams& p, const Shape& s, cudaStream_t stream) {
  if constexpr (sizeof(T) == 2) {
    if (s.kind == 3)
      return launch_shape(block_norm_bwd_kernel<T, GATE, FORM, SIMPLE, 2, 512>, p, s, stream);
  }
  return launch_shape(s.kind == 2   ? block_norm_bwd_kernel<T, GATE, FORM, SIMPLE, 1, 512>
                      : s.kind == 1 ? block_norm_bwd_kernel<T, GATE, FORM, SIMPLE, 2, 256>
                                    : block_norm_bwd_kernel<T, GATE, FORM, SIMPLE, 2, 128>,
                      p, s, stream);
}

template <typename T, bool GATE>
cudaError_t run_backward(const BlockNormParams& p, int num_sms, Shape* s, cudaStream_t stream) {
  if (!p.pre) {
    *s = backward_shape<T, GATE, false>(p.T, p.W, num_sms);
    return run_backward<T, GATE, kOutput, false>(p, *s, stream);
  }
  *s = backward_shape<T, GATE, true>(p.T, p.W, num_sms);
  if (!(p.post && p.G == p.W && p.residual && p.dy && p.dres))
    return run_backward<T, GATE, kAny, false>(p, *s, stream);
  return s->simple() ? run_backward<T, GATE, kBlock, true>(p, *s, stream)
                     : run_backward<T, GATE, kBlock, false>(p, *s, stream);
}

}  // namespace

template <typename T>
cudaError_t launch_block_norm_rows(const BlockNormParams& p, int num_sms, int* ctas, int* cluster,
                                   cudaStream_t stream) {
  Shape s = {};
  const cudaError_t e = p.gate ? run_backward<T, true>(p, num_sms, &s, stream)
                               : run_backward<T, false>(p, num_sms, &s, stream);
  *ctas = s.ctas;
  *cluster = s.cluster;
  return e;
}

template <typename T>
int block_norm_rows_ctas(int T_rows, int W, bool pre, int num_sms) {
  int most = 0;
  if (pre) {
    backward_shape<T, true, true>(T_rows, W, num_sms, &most);
    backward_shape<T, false, true>(T_rows, W, num_sms, &most);
  } else {
    backward_shape<T, true, false>(T_rows, W, num_sms, &most);
    backward_shape<T, false, false>(T_rows, W, num_sms, &most);
  }
  return most;
}

}  // namespace flare
