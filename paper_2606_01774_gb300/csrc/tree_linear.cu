// Gated delta rule along the paths of a drafted tree, on CUDA cores in fp32.
//
// Unrolling the recurrence along node i's path, with gamma_i the sum of the
// log-gates over the path and anc(i) the path's set:
//   A[i][j]  = beta_i exp(gamma_i - gamma_j) (k_i . k_j),   j in anc(i), j != i
//   delta    = (I + A)^{-1} diag(beta) (V - diag(exp gamma) K S0)
//   out_i    = scale (exp(gamma_i) S0^T q_i + sum_{j in anc(i)} exp(gamma_i - gamma_j) (q_i . k_j) delta_j)
// A is strictly lower triangular because parents come before their children,
// so the state S0 is read once for all nodes and no node's state is formed.
//
// One CTA per (request, value head).  Thread (part, c) owns value column c;
// the parts share the nodes in the products with S0, whose rows stream
// through registers, 16 ahead of their use, against keys and queries broadcast
// from shared memory.
// The Grams are built one (i, j) pair per thread.  Column c's substitution and
// readout need only its own deltas.
#include "common.cuh"
#include "kernels.h"
#include "tree.cuh"

namespace flare {

namespace {
constexpr int kParts = 4;
}

template <typename T, int DK, int DV>
__global__ void __launch_bounds__(kParts * DV) tree_linear_kernel(GdrParams p) {
  constexpr int kThreads = kParts * DV;
  constexpr int kPer = kMaxNodes / kParts;  // nodes per part
  constexpr int kKS = DK + 4;               // staged row stride: 16-byte rows over all banks
  extern __shared__ __align__(16) float sm[];
  __shared__ uint64_t anc[kMaxNodes];
  __shared__ float gam[kMaxNodes], bet[kMaxNodes], lg[kMaxNodes];
  __shared__ int tree_ok;
  const int r = blockIdx.x / p.Hv, j = blockIdx.x % p.Hv, h = j / (p.Hv / p.Hk);
  const int tid = threadIdx.x, c = tid % DV, part = tid / DV;
  const int n = p.node_len[r], slot = p.state_slot[r];
  int bad = 0;
  if (n < 0 || n > p.B) bad |= FLARE_DEV_BAD_TREE;
  if (slot < 0 || slot >= p.nslots) bad |= FLARE_DEV_BAD_SLOT;
  if (bad) {
    if (tid == 0) flag(p.dev_status, bad);
    return;
  }
  // the state's column c, 16 rows ahead of their use, the first ones from here on
  constexpr int kAhead = 16;
  const float* S = p.state_pool + ((size_t)slot * p.Hv + j) * DK * DV + c;
  float ahead[kAhead];
#pragma unroll
  for (int e = 0; e < kAhead; ++e) ahead[e] = S[(size_t)e * DV];
  if (tid < 32) {
    int p0, p1;
    const bool ok = warp_load_tree(p.parent + (size_t)r * p.B, n, p0, p1);
    if (ok) {
      uint64_t a0, a1;
      warp_paths(n, p0, p1, a0, a1);
      anc[tid] = a0;
      anc[tid + 32] = a1;
    }
    if (tid == 0) tree_ok = ok;
  } else if (tid < 32 + kMaxNodes) {
    const int i = tid - 32;
    const size_t g = ((size_t)r * p.B + i) * p.Hv + j;
    lg[i] = i < n ? p.log_decay[g] : 0.f;
    bet[i] = i < n ? p.beta[g] : 0.f;
  }
  float* Ks = sm;                       // [n][kKS]
  float* Qs = Ks + p.B * kKS;           // [n][kKS]
  float* A = Qs + p.B * kKS;            // [n][kMaxNodes]: beta e^(..) k.k below the diagonal
  float* M = A + p.B * kMaxNodes;       // [n][kMaxNodes]: e^(..) q.k
  float* X = M + p.B * kMaxNodes;       // [n][DV]: beta (v - e^gamma K S0), then delta
  float* Y = X + p.B * DV;              // [n][DV]: e^gamma S0^T q
  const T* k = static_cast<const T*>(p.k) + ((size_t)r * p.B * p.Hk + h) * DK;
  const T* q = static_cast<const T*>(p.q) + ((size_t)r * p.B * p.Hk + h) * DK;
  const T* v = static_cast<const T*>(p.v) + ((size_t)r * p.B * p.Hv + j) * DV;
  T* out = static_cast<T*>(p.out_causal) + ((size_t)r * p.B * p.Hv + j) * DV;
  constexpr int kE = 16 / sizeof(T);  // staged in 16-byte pieces
  for (int e = tid; e < n * (DK / kE); e += kThreads) {
    const int i = e / (DK / kE), d = e % (DK / kE) * kE;
    const uint4 kw = *reinterpret_cast<const uint4*>(k + (size_t)i * p.Hk * DK + d);
    const uint4 qw = *reinterpret_cast<const uint4*>(q + (size_t)i * p.Hk * DK + d);
#pragma unroll
    for (int x = 0; x < kE; ++x) {
      Ks[i * kKS + d + x] = to_f32(reinterpret_cast<const T*>(&kw)[x]);
      Qs[i * kKS + d + x] = to_f32(reinterpret_cast<const T*>(&qw)[x]);
    }
  }
  __syncthreads();
  if (!tree_ok) {
    if (tid == 0) flag(p.dev_status, FLARE_DEV_BAD_TREE);
    return;
  }
  if (tid < kMaxNodes) {
    float g = 0.f;  // ancestors in index order
    for (uint64_t a = tid < n ? anc[tid] : 0ull; a; a &= a - 1) g += lg[__ffsll((long long)a) - 1];
    gam[tid] = g;
  }
  __syncthreads();
  // the Grams
  for (int e = tid; e < n * n; e += kThreads) {
    const int i = e / n, m = e - i * n;
    if (!((anc[i] >> m) & 1)) {
      A[i * kMaxNodes + m] = M[i * kMaxNodes + m] = 0.f;
      continue;
    }
    float kk = 0.f, qk = 0.f;
#pragma unroll 4
    for (int d = 0; d < DK; d += 4) {
      const float4 b = *reinterpret_cast<const float4*>(Ks + m * kKS + d);
      const float4 a = *reinterpret_cast<const float4*>(Ks + i * kKS + d);
      const float4 w = *reinterpret_cast<const float4*>(Qs + i * kKS + d);
      kk = fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, fmaf(a.w, b.w, kk))));
      qk = fmaf(w.x, b.x, fmaf(w.y, b.y, fmaf(w.z, b.z, fmaf(w.w, b.w, qk))));
    }
    const float e2 = expf(gam[i] - gam[m]);
    A[i * kMaxNodes + m] = m == i ? 0.f : bet[i] * e2 * kk;
    M[i * kMaxNodes + m] = e2 * qk;
  }
  // K S0 and Q S0: this part's nodes, column c
  {
    const int n0 = part * kPer, n1 = min(n, n0 + kPer);
    float wk[kPer], wq[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) wk[i] = wq[i] = 0.f;
    if (n0 < n) {
#pragma unroll 1
      for (int d0 = 0; d0 < DK; d0 += kAhead) {
        float s[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
          s[e] = ahead[e];
          if (d0 + kAhead < DK) ahead[e] = S[(size_t)(d0 + kAhead + e) * DV];
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          if (n0 + i < n1) {
#pragma unroll
            for (int e = 0; e < kAhead; e += 4) {
              const float4 a = *reinterpret_cast<const float4*>(Ks + (n0 + i) * kKS + d0 + e);
              const float4 b = *reinterpret_cast<const float4*>(Qs + (n0 + i) * kKS + d0 + e);
              wk[i] = fmaf(a.x, s[e], fmaf(a.y, s[e + 1], fmaf(a.z, s[e + 2], fmaf(a.w, s[e + 3], wk[i]))));
              wq[i] = fmaf(b.x, s[e], fmaf(b.y, s[e + 1], fmaf(b.z, s[e + 2], fmaf(b.w, s[e + 3], wq[i]))));
            }
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (n0 + i < n1) {
        const int t = n0 + i;
        const float e = expf(gam[t]);
        X[t * DV + c] = bet[t] * (to_f32(v[(size_t)t * p.Hv * DV + c]) - e * wk[i]);
        Y[t * DV + c] = e * wq[i];
      }
    }
  }
  __syncthreads();
  if (part == 0) {  // delta = (I + A)^{-1} X, forward over the nodes
#pragma unroll 1
    for (int i = 1; i < n; ++i) {
      float x = X[i * DV + c];
#pragma unroll 4
      for (int m = 0; m < i; ++m) x = fmaf(-A[i * kMaxNodes + m], X[m * DV + c], x);
      X[i * DV + c] = x;
    }
  }
  __syncthreads();
  for (int i = part; i < p.B; i += kParts) {
    float y = 0.f;
    if (i < n) {
      y = Y[i * DV + c];
#pragma unroll 4
      for (int m = 0; m <= i; ++m) y = fmaf(M[i * kMaxNodes + m], X[m * DV + c], y);
    }
    out[(size_t)i * p.Hv * DV + c] = from_f32<T>(p.scale * y);
  }
}

namespace {

template <typename T, int DK, int DV>
cudaError_t launch_t(const GdrParams& p, cudaStream_t stream) {
  auto smem_for = [](int B) {
    return (int)sizeof(float) * B * (2 * (DK + 4) + 2 * kMaxNodes + 2 * DV);
  };
  cudaError_t e = cudaFuncSetAttribute(tree_linear_kernel<T, DK, DV>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       smem_for(kMaxNodes));
  if (e != cudaSuccess) return e;
  tree_linear_kernel<T, DK, DV>
      <<<(unsigned)((long)p.R * p.Hv), kParts * DV, smem_for(p.B), stream>>>(p);
  note_launches(1);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_d(const GdrParams& p, cudaStream_t stream) {
  if constexpr (sizeof(T) == 4)  // in bf16 that state takes the tensor cores
    if (p.dk == 128 && p.dv == 128) return launch_t<T, 128, 128>(p, stream);
  if (p.dk == 128 && p.dv == 64) return launch_t<T, 128, 64>(p, stream);
  if (p.dk == 64 && p.dv == 128) return launch_t<T, 64, 128>(p, stream);
  if (p.dk == 64 && p.dv == 64) return launch_t<T, 64, 64>(p, stream);
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_tree_linear(const GdrParams& p, bool bf16, cudaStream_t stream) {
  if (p.R == 0) return cudaSuccess;
  if (bf16 && tree_linear_tc_supported(p.dk, p.dv)) return launch_tree_linear_tc(p, stream);
  return bf16 ? launch_d<__nv_bfloat16>(p, stream) : launch_d<float>(p, stream);
}

}  // namespace flare
