// Block norms, forward (block_norm.cuh has the formulas), and the last step of their weight
// gradients.
#include "block_norm.cuh"
#include "pdl.cuh"

namespace flare {

namespace {

constexpr int kThreads = 1024;  // of the largest CTA, eight elements each

// A thread's own places in shared memory: its eight elements of each input of a row.
template <typename T>
struct Slots {
  static constexpr int M = 8 / Piece<T>::N;
  uint4* at;   // of this thread, piece 0
  int pieces;  // from one piece to the next: threads of the CTA

  __device__ __forceinline__ void fetch(int array, const T* src, const bool (&mine)[M]) const {
#pragma unroll
    for (int i = 0; i < M; ++i)
      if (mine[i]) cp_async16(at + (array * M + i) * pieces, src + i * kFar);
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

  template <typename T>
  __device__ __forceinline__ void fill(const BlockNormParams& p, int c,
                                       const bool (&mine)[kHalves<T>]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (!mine[i % kHalves<T>]) continue;
      const int at_w = c + weight_column<T>(i);
      float4 w = make_float4(1.f, 1.f, 1.f, 1.f);
      if (p.wpost) w = *reinterpret_cast<const float4*>(p.wpost + (p.shared ? at_w % p.G : at_w));
      w.x *= p.alpha, w.y *= p.alpha, w.z *= p.alpha, w.w *= p.alpha;
      reinterpret_cast<float4*>(at)[i * pieces] = w;
      w = make_float4(1.f, 1.f, 1.f, 1.f);
      if (p.wpre) w = *reinterpret_cast<const float4*>(p.wpre + at_w);
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

}  // namespace

template <typename T, bool GATE, bool SIMPLE>
__global__ void __launch_bounds__(kThreads, 1)
    block_norm_kernel(const __grid_constant__ BlockNormParams p, const __grid_constant__ Shape s) {
  extern __shared__ __align__(16) char smem[];
  __shared__ float buf[2][2][kMaxWarps], far[2][2][kMaxCluster];
  const int thread = threadIdx.y * blockDim.x + threadIdx.x;
  const int threads = blockDim.x * blockDim.y;
  const int rank = blockIdx.x % s.cluster;
  RowSum<SIMPLE> row_sum{buf, far, s.cluster, rank, 0};
  const int at_row = first_column<T>(0), c = rank * s.cols + at_row;
  bool mine[kHalves<T>];
#pragma unroll
  for (int i = 0; i < kHalves<T>; ++i)
    mine[i] = at_row + i * kFar < s.cols && c + i * kFar < p.W;
  const bool heads = p.post && p.G != p.W;
  const float per_group = 1.f / (float)p.G, per_row = 1.f / (float)p.W;
  const Weights weights{reinterpret_cast<uint4*>(smem) + thread, threads};
  uint4* ring = reinterpret_cast<uint4*>(smem) + 4 * threads + thread;
  const int stage = s.arrays * Slots<T>::M * threads;
  constexpr int kGate = 1, kRes = 1 + GATE;

  if (!mine[kHalves<T> - 1]) {  // columns past the row's hold zeros throughout
#pragma unroll 1
    for (int i = 0; i < 4 + s.stages * s.arrays * Slots<T>::M; ++i)
      weights.at[i * threads] = make_uint4(0, 0, 0, 0);
  }
  if (s.cluster > 1) cluster_sync();  // every CTA runs before another writes to its memory
  const int64_t step = (int64_t)(gridDim.x / s.cluster) * blockDim.y;
  const int64_t first = (int64_t)(blockIdx.x / s.cluster) * blockDim.y + threadIdx.y;
  const auto fetch = [&](int64_t row, int at) {
    if (row < p.T) {
      const Slots<T> to{ring + at * stage, threads};
      to.fetch(0, static_cast<const T*>(p.x) + row * p.x_stride + c, mine);
      if (GATE) to.fetch(kGate, static_cast<const T*>(p.gate) + row * p.gate_stride + c, mine);
      if (p.residual) to.fetch(kRes, static_cast<const T*>(p.residual) + row * p.W + c, mine);
    }
    cp_async_commit();
  };
  for (int i = 0; i < s.stages - 1; ++i) fetch(first + i * step, i);
  weights.fill<T>(p, c, mine);  // behind the first rows
  int at = 0;
  for (int64_t row = first; row < p.T; row += step) {
    const int last = at == 0 ? s.stages - 1 : at - 1;
    fetch(row + (s.stages - 1) * step, last);
    wait_rows(s.stages - 1);
    const Slots<T> in{ring + at * stage, threads};
    at = at + 1 == s.stages ? 0 : at + 1;

    uint64_t y[4], t[4] = {}, w[4];
    in.read(0, y);
    weights.read(0, w);
    if (p.post) {
      float sum[2];
      if (heads) {
        group_sums<T>(y, y, p.G, sum);
      } else {
        float all[1] = {dot8(y, y)};
        row_sum(all);
        sum[0] = sum[1] = all[0];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = f2_mul(w[i], f2_dup(rsqrtf(sum[i / 2] * per_group + p.eps)));
    }
    if (GATE) {
      uint64_t sig[4] = {};
      in.read(kGate, t);
      sigmoid8<T>(p.act, t, sig);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = f2_mul(w[i], activation(p.act, t[i], sig[i]));
        t[i] = 0;
      }
    }
    if (p.residual) in.read(kRes, t);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = f2_fma(y[i], w[i], t[i]);
    if (p.y) store_row<T>(static_cast<T*>(p.y) + row * p.W + c, y, mine);
    if (p.pre) {
      float squares[1] = {dot8(y, y)};
      row_sum(squares);
      const uint64_t r = f2_dup(rsqrtf(squares[0] * per_row + p.eps));
      weights.read(1, w);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = f2_mul(y[i], f2_mul(w[i], r));
      store_row<T>(static_cast<T*>(p.h) + row * p.W + c, y, mine);
    }
  }
  if (s.cluster > 1) cluster_sync();  // none leaves while another may write to its memory
}

// The CTAs' weight gradients joined: 32 columns a CTA, its warps one partial sum in 32 (or 16) each,
// 16 of them in flight, added in order at the end: the same bits every time, which atomics would
// not give.  3 to 8 us behind the rows, started while their last CTAs finish.
__global__ void __launch_bounds__(1024)
    block_norm_weights_kernel(const __grid_constant__ BlockNormParams p, int ctas, int cluster) {
  constexpr int kInFlight = 16;
  __shared__ float buf[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
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
    for (int i0 = warp; i0 < n; i0 += warps * kInFlight) {
      float part[kInFlight];
#pragma unroll
      for (int k = 0; k < kInFlight; ++k)
        part[k] = i0 + warps * k < n ? at[(int64_t)(i0 + warps * k) * wide] : 0.f;
#pragma unroll
      for (int k = 0; k < kInFlight; ++k) sum += part[k];
    }
  }
  buf[warp][lane] = sum;
  __syncthreads();
  for (int col = warp; col < 32; col += warps) {
    sum = warp_sum(lane < warps ? buf[lane][col] : 0.f);
    if (lane == 0 && blockIdx.x * 32 + col < wide) out[blockIdx.x * 32 + col] = sum;
  }
}

namespace {

template <typename T>
cudaError_t run_forward(const BlockNormParams& p, int num_sms, cudaStream_t stream) {
  // small CTAs where a row needs no more: 32 warps an SM in all
  const int arrays = 1 + (p.gate != nullptr) + (p.residual != nullptr);
  const int per_thread = 64 + 2 * 8 * (int)sizeof(T) * arrays;  // weights and two rows
  int most = p.W <= 2048 ? 256 : p.W <= 4096 ? 512 : kThreads;
  while (most > 512 && most * per_thread + kSmemOwn > kSmemMost) most /= 2;
  Shape s = teams_for(p.T, p.W, 1, most, num_sms);
  s.arrays = arrays;
  const int threads = s.team * s.teams;
  const int per_sm = threads > 512 ? 1 : threads > 256 ? 2 : threads > 128 ? 4 : 8;
  // as many rows as there is room for
  const int own = threads * 64, row = threads * 8 * (int)sizeof(T) * arrays;
  s.stages = 2;
  while (s.stages < 4 && own + row * (s.stages + 1) + kSmemOwn <= kSmem / per_sm) ++s.stages;
  s.smem = own + row * s.stages;
  const int room = kSmem / (s.smem + kSmemOwn);
  set_ctas(s, p.T, room < per_sm ? room : per_sm, num_sms);
  if (s.simple())
    return launch_shape(p.gate ? block_norm_kernel<T, true, true> : block_norm_kernel<T, false, true>,
                        p, s, stream);
  return launch_shape(p.gate ? block_norm_kernel<T, true, false> : block_norm_kernel<T, false, false>,
                      p, s, stream);
}

}  // namespace

cudaError_t launch_block_norm(const BlockNormParams& p, bool bf16, int num_sms,
                              cudaStream_t stream) {
  if (p.T == 0) return cudaSuccess;
  note_launches(1);
  return bf16 ? run_forward<__nv_bfloat16>(p, num_sms, stream)
              : run_forward<float>(p, num_sms, stream);
}

int block_norm_bwd_ctas(int T, int W, bool pre, bool bf16, int num_sms) {
  if (T == 0) return 0;
  return bf16 ? block_norm_rows_ctas<__nv_bfloat16>(T, W, pre, num_sms)
              : block_norm_rows_ctas<float>(T, W, pre, num_sms);
}

cudaError_t launch_block_norm_bwd(const BlockNormParams& p, bool bf16, int num_sms,
                                  cudaStream_t stream) {
  const bool weights = p.dwpost || p.dwpre;
  if (p.T == 0 && !weights) return cudaSuccess;
  int ctas = 0, cluster = 1;
  if (p.T > 0) {
    note_launches(1);
    const cudaError_t e =
        bf16 ? launch_block_norm_rows<__nv_bfloat16>(p, num_sms, &ctas, &cluster, stream)
             : launch_block_norm_rows<float>(p, num_sms, &ctas, &cluster, stream);
    if (e != cudaSuccess) return e;
  }
  if (weights) {  // of no rows: zeros
    note_launches(1);
    // 16 warps where they take all sums at once, or where CTAs of 32 are more than the SMs hold (300
    // rows of 6000: 13.8 us, 14.3; 150 of 8192: 13.3, 15.0), 32 for many sums of few columns (1021
    // fp32 rows of 16 heads: 19.4 us, 19.7)
    const bool few = ctas / cluster <= 16 * 16 || (p.W + 31) / 32 * 2 > num_sms;
    const int threads = few ? 512 : 1024;
    return pdl_launch(block_norm_weights_kernel, dim3((unsigned)(p.W + 31) / 32, 2), threads, 0,
                      stream, p.T > 0, 1, p, ctas, cluster);
  }
  return cudaSuccess;
}

}  // namespace flare
