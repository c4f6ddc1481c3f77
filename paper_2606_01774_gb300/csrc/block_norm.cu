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
// A CTA takes a row at a time and keeps it in registers, eight elements of a thread next to
// each other, from the one time it is read to the outputs: bound by bytes.  The gradient of a weight
// is summed over a CTA's rows in registers, the CTAs' sums in a fixed order by a second kernel.
#include "common.cuh"
#include "kernels.h"
#include "piece.cuh"

namespace flare {

namespace {

template <typename T>
struct Eight {  // eight elements as they lie in memory
  static constexpr int M = 8 / Piece<T>::N;
  uint4 u[M];
  __device__ __forceinline__ void read(const T* p) {
#pragma unroll
    for (int i = 0; i < M; ++i) u[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void values(float* x) const {
#pragma unroll
    for (int i = 0; i < M; ++i) Piece<T>::load(u[i], x + i * Piece<T>::N);
  }
};

template <typename T>
__device__ __forceinline__ void write8(T* p, const float* x) {
#pragma unroll
  for (int i = 0; i < Eight<T>::M; ++i)
    reinterpret_cast<uint4*>(p)[i] = Piece<T>::store(x + i * Piece<T>::N);
}

__device__ __forceinline__ void weight8(const float* w, int at, float* out) {
  const float4 a = *reinterpret_cast<const float4*>(w + at);
  const float4 b = *reinterpret_cast<const float4*>(w + at + 4);
  out[0] = a.x, out[1] = a.y, out[2] = a.z, out[3] = a.w;
  out[4] = b.x, out[5] = b.y, out[6] = b.z, out[7] = b.w;
}

// Sums over the CTA, the same in every thread; `slot` alternates between calls.
template <int K>
__device__ __forceinline__ void cta_sum(float (&v)[K], float (*buf)[K][32]) {
  const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = warp_sum(v[k]);
  if (warps == 1) return;
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) (*buf)[k][threadIdx.x >> 5] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = warp_sum(lane < warps ? (*buf)[k][lane] : 0.f);
}

// Sum over `lanes` neighbouring lanes.
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The gate's activation and its derivative.
__device__ __forceinline__ float act(int kind, float z, float& slope) {
  if (kind == FLARE_ACT_NONE) {
    slope = 1.f;
    return z;
  }
  const float a = 1.f / (1.f + expf(-z));
  if (kind == FLARE_ACT_SIGMOID) {
    slope = a * (1.f - a);
    return a;
  }
  slope = a * (1.f + z * (1.f - a));
  return z * a;
}

}  // namespace

template <typename T, int V>
__global__ void __launch_bounds__(512) block_norm_kernel(const __grid_constant__ BlockNormParams p) {
  __shared__ float buf[2][1][32];
  const int tid = threadIdx.x, W = p.W;
  const bool heads = p.post && p.G != W;
  const float per_group = 1.f / (float)p.G, per_row = 1.f / (float)W;
  for (int row = blockIdx.x; row < p.T; row += gridDim.x) {
    const T* x_row = static_cast<const T*>(p.x) + (int64_t)row * p.x_stride;
    const T* g_row = static_cast<const T*>(p.gate) + (int64_t)row * p.gate_stride;
    const T* r_row = static_cast<const T*>(p.residual) + (int64_t)row * W;
    Eight<T> xin[V], gin[V], rin[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * blockDim.x + tid) * 8;
      if (c < W) {
        xin[j].read(x_row + c);
        if (p.gate) gin[j].read(g_row + c);
        if (p.residual) rin[j].read(r_row + c);
      }
    }
    float q[V], y[V][8];
    if (p.post) {
      float all[1] = {0.f};
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float x[8], s = 0.f;
        if ((j * blockDim.x + tid) * 8 < W) {
          xin[j].values(x);
#pragma unroll
          for (int e = 0; e < 8; ++e) s += x[e] * x[e];
        }
        if (heads) q[j] = rsqrtf(lanes_sum(s, p.G / 8) * per_group + p.eps);
        else all[0] += s;
      }
      if (!heads) {
        cta_sum<1>(all, &buf[0]);
#pragma unroll
        for (int j = 0; j < V; ++j) q[j] = rsqrtf(all[0] * per_group + p.eps);
      }
    }
    float squares[1] = {0.f};
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * blockDim.x + tid) * 8;
      if (c >= W) continue;
      xin[j].values(y[j]);
      if (p.post) {
        float w[8];
        if (p.wpost) weight8(p.wpost, p.shared ? c % p.G : c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[j][e] *= p.wpost ? q[j] * w[e] : q[j];
      }
      if (p.gate) {
        float z[8], slope;
        gin[j].values(z);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[j][e] *= act(p.act, z[e], slope);
      }
      float res[8];
      if (p.residual) rin[j].values(res);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[j][e] = p.alpha * y[j][e] + (p.residual ? res[e] : 0.f);
        squares[0] += y[j][e] * y[j][e];
      }
      if (p.y) write8<T>(static_cast<T*>(p.y) + (int64_t)row * W + c, y[j]);
    }
    if (p.pre) {
      cta_sum<1>(squares, &buf[1]);
      const float r = rsqrtf(squares[0] * per_row + p.eps);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int c = (j * blockDim.x + tid) * 8;
        if (c >= W) continue;
        float w[8];
        if (p.wpre) weight8(p.wpre, c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[j][e] *= p.wpre ? r * w[e] : r;
        write8<T>(static_cast<T*>(p.h) + (int64_t)row * W + c, y[j]);
      }
    }
    if (blockDim.x > 32) __syncthreads();  // the sums' buffers before the next row's
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(512)
    block_norm_bwd_kernel(const __grid_constant__ BlockNormParams p) {
  __shared__ float buf1[1][32], buf2[2][32], buf3[1][32];
  const int tid = threadIdx.x, W = p.W;
  const bool heads = p.post && p.G != W;
  const float per_group = 1.f / (float)p.G, per_row = 1.f / (float)W;
  float dwpost[V][8], dwpre[V][8];
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) dwpost[j][e] = dwpre[j][e] = 0.f;

  for (int row = blockIdx.x; row < p.T; row += gridDim.x) {
    Eight<T> xin[V], gin[V], rin[V], yin[V], hin[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * blockDim.x + tid) * 8;
      if (c < W) {
        const int64_t at = (int64_t)row * W + c;
        xin[j].read(static_cast<const T*>(p.x) + (int64_t)row * p.x_stride + c);
        if (p.gate) gin[j].read(static_cast<const T*>(p.gate) + (int64_t)row * p.gate_stride + c);
        if (p.pre && p.residual) rin[j].read(static_cast<const T*>(p.residual) + at);
        if (p.dy) yin[j].read(static_cast<const T*>(p.dy) + at);
        if (p.pre) hin[j].read(static_cast<const T*>(p.dh) + at);
      }
    }
    float q[V];
    if (p.post) {
      float all[1] = {0.f};
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float x[8], s = 0.f;
        if ((j * blockDim.x + tid) * 8 < W) {
          xin[j].values(x);
#pragma unroll
          for (int e = 0; e < 8; ++e) s += x[e] * x[e];
        }
        if (heads) q[j] = rsqrtf(lanes_sum(s, p.G / 8) * per_group + p.eps);
        else all[0] += s;
      }
      if (!heads) {
        cta_sum<1>(all, &buf1);
#pragma unroll
        for (int j = 0; j < V; ++j) q[j] = rsqrtf(all[0] * per_group + p.eps);
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) q[j] = 1.f;
    }

    float g[V][8];  // the gradient at y
    float sums[2] = {0.f, 0.f};
    if (p.pre) {
      float y[V][8];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int c = (j * blockDim.x + tid) * 8;
        if (c >= W) continue;
        float w[8], t[8], slope;
        xin[j].values(y[j]);
        if (p.post) {
          if (p.wpost) weight8(p.wpost, p.shared ? c % p.G : c, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[j][e] *= p.wpost ? q[j] * w[e] : q[j];
        }
        if (p.gate) {
          gin[j].values(t);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[j][e] *= act(p.act, t[e], slope);
        }
        if (p.residual) rin[j].values(t);
        hin[j].values(g[j]);
        if (p.wpre) weight8(p.wpre, c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y[j][e] = p.alpha * y[j][e] + (p.residual ? t[e] : 0.f);
          sums[0] += y[j][e] * y[j][e];
          sums[1] += y[j][e] * (p.wpre ? g[j][e] * w[e] : g[j][e]);
        }
      }
      cta_sum<2>(sums, &buf2);
      const float r = rsqrtf(sums[0] * per_row + p.eps);
      const float back = sums[1] * per_row * r * r;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int c = (j * blockDim.x + tid) * 8;
        if (c >= W) continue;
        float w[8], t[8];
        if (p.wpre) weight8(p.wpre, c, w);
        if (p.dy) yin[j].values(t);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          dwpre[j][e] += g[j][e] * y[j][e] * r;
          g[j][e] = r * ((p.wpre ? g[j][e] * w[e] : g[j][e]) - y[j][e] * back);
          if (p.dy) g[j][e] += t[e];
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if ((j * blockDim.x + tid) * 8 < W) yin[j].values(g[j]);
    }

    float dot[V], all[1] = {0.f};
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * blockDim.x + tid) * 8;
      dot[j] = 0.f;
      if (c < W) {
        if (p.dres) write8<T>(static_cast<T*>(p.dres) + (int64_t)row * W + c, g[j]);
        float x[8], w[8], z[8], slope, dz[8];
        xin[j].values(x);
        if (p.post && p.wpost) weight8(p.wpost, p.shared ? c % p.G : c, w);
        if (p.gate) gin[j].values(z);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float d = p.alpha * g[j][e];
          const float xq = x[e] * q[j];
          if (p.gate) {
            const float a = act(p.act, z[e], slope);
            dz[e] = d * (p.post && p.wpost ? xq * w[e] : xq) * slope;
            d *= a;
          }
          if (p.post) {
            dwpost[j][e] += d * xq;
            if (p.wpost) d *= w[e];
            dot[j] += x[e] * d;
          }
          g[j][e] = d;
        }
        if (p.gate)
          write8<T>(static_cast<T*>(p.dgate) + (int64_t)row * p.gate_stride + c, dz);
      }
      if (heads) dot[j] = lanes_sum(dot[j], p.G / 8);
      else all[0] += dot[j];
    }
    if (p.post && !heads) {
      cta_sum<1>(all, &buf3);
#pragma unroll
      for (int j = 0; j < V; ++j) dot[j] = all[0];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * blockDim.x + tid) * 8;
      if (c >= W) continue;
      if (p.post) {
        float x[8];
        xin[j].values(x);
        const float back = dot[j] * per_group * q[j] * q[j];
#pragma unroll
        for (int e = 0; e < 8; ++e) g[j][e] = q[j] * (g[j][e] - x[e] * back);
      }
      write8<T>(static_cast<T*>(p.dx) + (int64_t)row * p.x_stride + c, g[j]);
    }
    if (blockDim.x > 32) __syncthreads();
  }

  if (!p.part) return;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int c = (j * blockDim.x + tid) * 8;
    if (c >= W) continue;
    float* at = p.part + (int64_t)blockIdx.x * 2 * W + c;
    write8<float>(at, dwpost[j]);
    write8<float>(at + W, dwpre[j]);
  }
}

// The CTAs' partial weight gradients joined: 32 columns a CTA, eight warps that take every eighth
// CTA (and group) and are then added in order.
__global__ void __launch_bounds__(256)
    block_norm_weights_kernel(const __grid_constant__ BlockNormParams p, int ctas) {
  __shared__ float buf[8][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool post = blockIdx.y == 0;
  float* out = post ? p.dwpost : p.dwpre;
  const int wide = post && p.shared ? p.G : p.W, c = blockIdx.x * 32 + lane;
  if (!out || blockIdx.x * 32 >= wide) return;
  const int groups = p.W / wide;
  float sum = 0.f;
  if (c < wide) {
    const float* at = p.part + (post ? 0 : p.W) + c;
    for (int i = warp; i < ctas * groups; i += 8) {
      const int cta = i / groups;
      sum += at[(int64_t)cta * 2 * p.W + (i - cta * groups) * wide];
    }
  }
  buf[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && c < wide) {
    for (int k = 1; k < 8; ++k) sum += buf[k][lane];
    out[c] = sum;
  }
}

namespace {

int row_threads(int W, int V) { return (W + 8 * V * 32 - 1) / (8 * V * 32) * 32; }
int vectors(int W) { return W <= 2048 ? 1 : W <= 8192 ? 2 : 4; }

template <typename T>
void run(const BlockNormParams& p, bool bwd, int ctas, cudaStream_t stream) {
  const int v = vectors(p.W), threads = row_threads(p.W, v);
  const auto go = [&](auto* fwd_kernel, auto* bwd_kernel) {
    if (bwd) bwd_kernel<<<ctas, threads, 0, stream>>>(p);
    else fwd_kernel<<<ctas, threads, 0, stream>>>(p);
  };
  if (v == 1) go(block_norm_kernel<T, 1>, block_norm_bwd_kernel<T, 1>);
  else if (v == 2) go(block_norm_kernel<T, 2>, block_norm_bwd_kernel<T, 2>);
  else go(block_norm_kernel<T, 4>, block_norm_bwd_kernel<T, 4>);
}

}  // namespace

cudaError_t launch_block_norm(const BlockNormParams& p, bool bf16, int num_sms,
                              cudaStream_t stream) {
  if (p.T == 0) return cudaSuccess;
  const int ctas = p.T < 8 * num_sms ? p.T : 8 * num_sms;
  if (bf16) run<__nv_bfloat16>(p, false, ctas, stream);
  else run<float>(p, false, ctas, stream);
  note_launches(1);
  return cudaGetLastError();
}

int block_norm_bwd_ctas(int T, int W, bool bf16, int num_sms) {
  const int most = (W <= 2048 ? 4 : 2) * num_sms;
  return T < most ? T : most;
}

cudaError_t launch_block_norm_bwd(const BlockNormParams& p, bool bf16, int num_sms,
                                  cudaStream_t stream) {
  const int ctas = block_norm_bwd_ctas(p.T, p.W, bf16, num_sms);
  const bool weights = p.dwpost || p.dwpre;
  if (ctas == 0 && !weights) return cudaSuccess;
  if (ctas > 0) {
    if (bf16) run<__nv_bfloat16>(p, true, ctas, stream);
    else run<float>(p, true, ctas, stream);
    note_launches(1);
  }
  if (weights) {  // of no rows: zeros
    block_norm_weights_kernel<<<dim3((unsigned)(p.W + 31) / 32, 2), 256, 0, stream>>>(p, ctas);
    note_launches(1);
  }
  return cudaGetLastError();
}

}  // namespace flare
