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
// One CTA per (request, value head).  The state goes to shared memory whole, all of
// its reads in flight at once.  In the products with it a thread holds four value
// columns of two nodes, so that each piece read from shared memory serves several
// products; the substitution and the readout go over the nodes in fours.
// The FMA pipes and shared memory bound it.  64 requests x 32 heads: 16 nodes of
// 64 x 64 bf16 39.0 us (1.2 TB/s), of 64 x 64 fp32 39.6 us, of 128 x 128 fp32 124 us
// (1.5 TB/s); 64 nodes of 64 x 64 bf16 236 us; 8 requests x 16 nodes 19.2 us in fp32.
#include "async.cuh"
#include "common.cuh"
#include "kernels.h"
#include "tree.cuh"

namespace flare {

namespace {
constexpr int kParts = 4;  // threads per value column

// Floats of the staged state, which the two tables of the tree later take over.
__host__ __device__ constexpr int linear_state(int dk, int dv, int rows) {
  return dk * dv > 2 * rows * (kMaxNodes + 4) ? dk * dv : 2 * rows * (kMaxNodes + 4);
}
}  // namespace

// Threads hold their columns of up to NODES nodes in registers.
template <typename T, int DK, int DV, int NODES>
__global__ void __launch_bounds__(kParts * DV, NODES == 16 ? 256 / DV : DV == 64 ? 3 : 1)
    tree_linear_kernel(GdrParams p) {
  constexpr int kThreads = kParts * DV;
  constexpr int kGroups = DV / 4;               // column groups
  constexpr int kTeams = kThreads / kGroups;    // of threads with all columns: 16
  constexpr int kKS = DK + 4, kAS = kMaxNodes + 4;  // row strides: 16-byte rows over all banks
  constexpr int kXS = DV + 8;                       // eight columns of four rows in 32 banks
  extern __shared__ __align__(16) float sm[];
  __shared__ uint64_t anc[kMaxNodes];
  __shared__ float gam[kMaxNodes], bet[kMaxNodes];
  __shared__ int tree_ok;
  const int r = blockIdx.x / p.Hv, j = blockIdx.x % p.Hv, h = j / (p.Hv / p.Hk);
  const int tid = threadIdx.x;
  const int n = p.node_len[r], slot = p.state_slot[r];
  int bad = 0;
  if (n < 0 || n > p.B) bad |= FLARE_DEV_BAD_TREE;
  if (slot < 0 || slot >= p.nslots) bad |= FLARE_DEV_BAD_SLOT;
  if (bad) {
    if (tid == 0) flag(p.dev_status, bad);
    return;
  }
  const int rows = (p.B + 3) & ~3;
  float* S = sm;                          // [DK][DV]: the state
  float* Ks = S + linear_state(DK, DV, rows);   // [rows][kKS]
  float* Qs = Ks + rows * kKS;            // [rows][kKS]
  float* X = Qs + rows * kKS;             // [rows][kXS]: beta (v - e^gamma K S0)
  float* Y = X + rows * kXS;              // [rows][kXS]: e^gamma S0^T q, then the readout
  float* A = S;                           // [rows][kAS]: beta e^(..) k.k below the diagonal,
  float* M = A + rows * kAS;              // [rows][kAS]: e^(..) q.k; over the state, read by then
  const float* state = p.state_pool + ((size_t)slot * p.Hv + j) * DK * DV;
  for (int e = tid; e < DK * DV / 4; e += kThreads) cp_async16(S + 4 * e, state + 4 * e);
  cp_async_commit();
  if (tid < 32) {
    const size_t g = (size_t)r * p.B * p.Hv + j;
    float x0 = tid < n ? tree_log_gate(p.log_decay[g + (size_t)tid * p.Hv]) : 0.f;
    float x1 = tid + 32 < n ? tree_log_gate(p.log_decay[g + (size_t)(tid + 32) * p.Hv]) : 0.f;
    bet[tid] = tid < n ? p.beta[g + (size_t)tid * p.Hv] : 0.f;
    bet[tid + 32] = tid + 32 < n ? p.beta[g + (size_t)(tid + 32) * p.Hv] : 0.f;
    int p0, p1;
    const bool ok = warp_load_tree(p.parent + (size_t)r * p.B, n, p0, p1);
    if (ok) {
      uint64_t a0, a1;
      warp_paths<kMaxNodes>(n, p0, p1, a0, a1, x0, x1);
      anc[tid] = a0;
      anc[tid + 32] = a1;
      gam[tid] = x0;
      gam[tid + 32] = x1;
    }
    if (tid == 0) tree_ok = ok;
  }
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
  cp_async_wait<0>();
  __syncthreads();
  if (!tree_ok) {
    if (tid == 0) flag(p.dev_status, FLARE_DEV_BAD_TREE);
    return;
  }
  // K S0 and Q S0: nodes team, team + 16, ... two at a time, columns 4 cg .. 4 cg + 3
  const int cg = tid % kGroups, team = tid / kGroups;
#pragma unroll 1
  for (int t0 = team; t0 < n; t0 += 2 * kTeams) {
    const bool two = NODES > kTeams && n > kTeams;  // one tree's threads agree
    const int t1 = t0 + kTeams < n ? t0 + kTeams : t0;
    float4 w[4] = {};
    auto rows4 = [&](int t, const float* F, const float4 (&s)[4], int d, float4& o) {
      const float4 f = *reinterpret_cast<const float4*>(F + t * kKS + d);
      auto row = [&o](float x, const float4& r) {
        o.x = fmaf(x, r.x, o.x);
        o.y = fmaf(x, r.y, o.y);
        o.z = fmaf(x, r.z, o.z);
        o.w = fmaf(x, r.w, o.w);
      };
      row(f.x, s[0]);
      row(f.y, s[1]);
      row(f.z, s[2]);
      row(f.w, s[3]);
    };
#pragma unroll 2
    for (int d = 0; d < DK; d += 4) {
      float4 s[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s[e] = *reinterpret_cast<const float4*>(S + (d + e) * DV + 4 * cg);
      rows4(t0, Ks, s, d, w[0]);
      rows4(t0, Qs, s, d, w[1]);
      if (two) {
        rows4(t1, Ks, s, d, w[2]);
        rows4(t1, Qs, s, d, w[3]);
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int t = t0 + x * kTeams;
      if (t >= n) break;
      const float e = expf(gam[t]), b = bet[t];
      const float4 wk = w[2 * x], wq = w[2 * x + 1];
      const T* vt = v + (size_t)t * p.Hv * DV + 4 * cg;
      *reinterpret_cast<float4*>(X + t * kXS + 4 * cg) =
          make_float4(b * (to_f32(vt[0]) - e * wk.x), b * (to_f32(vt[1]) - e * wk.y),
                      b * (to_f32(vt[2]) - e * wk.z), b * (to_f32(vt[3]) - e * wk.w));
      *reinterpret_cast<float4*>(Y + t * kXS + 4 * cg) =
          make_float4(e * wq.x, e * wq.y, e * wq.z, e * wq.w);
    }
  }
  __syncthreads();  // the state has been read
  // the Grams: four nodes i by one m and a quarter of the dimensions per thread (a
  // key row read serves four pairs), the quarters joined by shuffles; zero outside
  // the paths and in the rows that fill up the last four
  const int n4 = (n + 3) & ~3, n8 = (n + 7) & ~7;
  for (int e = tid; e < n4 * n8; e += kThreads) {  // whole warps: 32 divides both
    const int quarter = e >> 3 & 3, i0 = e / (4 * n8) * 4;
    const int m = (e % (4 * n8) >> 5) * 8 + (e & 7);
    float kk[4] = {}, qk[4] = {};
    if (m < i0 + 4) {
#pragma unroll 2
      for (int d = 4 * quarter; d < DK; d += 16) {
        const float4 b = *reinterpret_cast<const float4*>(Ks + m * kKS + d);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float4 a = *reinterpret_cast<const float4*>(Ks + (i0 + x) * kKS + d);
          const float4 w = *reinterpret_cast<const float4*>(Qs + (i0 + x) * kKS + d);
          kk[x] = fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, fmaf(a.w, b.w, kk[x]))));
          qk[x] = fmaf(w.x, b.x, fmaf(w.y, b.y, fmaf(w.z, b.z, fmaf(w.w, b.w, qk[x]))));
        }
      }
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      kk[x] += __shfl_xor_sync(~0u, kk[x], 8);
      qk[x] += __shfl_xor_sync(~0u, qk[x], 8);
      kk[x] += __shfl_xor_sync(~0u, kk[x], 16);
      qk[x] += __shfl_xor_sync(~0u, qk[x], 16);
    }
    const int i = i0 + quarter;  // this lane's of the four
    const float ks = quarter < 2 ? (quarter ? kk[1] : kk[0]) : (quarter == 3 ? kk[3] : kk[2]);
    const float qs = quarter < 2 ? (quarter ? qk[1] : qk[0]) : (quarter == 3 ? qk[3] : qk[2]);
    const bool on = i < n && ((anc[i] >> m) & 1);
    const float g = on ? expf(gam[i] - gam[m]) : 0.f;
    A[i * kAS + m] = on && m != i ? bet[i] * g * ks : 0.f;
    M[i * kAS + m] = on ? g * qs : 0.f;
  }
  __syncthreads();
  // delta = (I + A)^{-1} X and the readout, four nodes at a time: four neighbouring
  // lanes hold one column, lane x of them nodes x, x + 4, ...; the four deltas of a
  // step go around by shuffles and from there into the later nodes
  const int col = tid / 4, sub = tid % 4;
  float x[NODES / 4], y[NODES / 4];
#pragma unroll
  for (int s = 0; s < NODES / 4; ++s) {
    const int i = 4 * s + sub;
    x[s] = i < n ? X[i * kXS + col] : 0.f;
    y[s] = i < n ? Y[i * kXS + col] : 0.f;
  }
#pragma unroll
  for (int b = 0; b < NODES / 4; ++b) {
    if (4 * b < n) {
      const float4 a = *reinterpret_cast<const float4*>(A + (4 * b + sub) * kAS + 4 * b);
      float d[4];  // A is zero on and above the diagonal
      d[0] = __shfl_sync(~0u, x[b], 0, 4);
      x[b] = fmaf(-a.x, d[0], x[b]);
      d[1] = __shfl_sync(~0u, x[b], 1, 4);
      x[b] = fmaf(-a.y, d[1], x[b]);
      d[2] = __shfl_sync(~0u, x[b], 2, 4);
      x[b] = fmaf(-a.z, d[2], x[b]);
      d[3] = __shfl_sync(~0u, x[b], 3, 4);
#pragma unroll
      for (int s = b; s < NODES / 4; ++s) {
        if (4 * s < n) {
          const int at = (4 * s + sub) * kAS + 4 * b;
          const float4 w = *reinterpret_cast<const float4*>(M + at);
          y[s] = fmaf(w.w, d[3], fmaf(w.z, d[2], fmaf(w.y, d[1], fmaf(w.x, d[0], y[s]))));
          if (s > b) {
            const float4 u = *reinterpret_cast<const float4*>(A + at);
            x[s] = fmaf(-u.w, d[3], fmaf(-u.z, d[2], fmaf(-u.y, d[1], fmaf(-u.x, d[0], x[s]))));
          }
        }
      }
    }
  }
#pragma unroll
  for (int s = 0; s < NODES / 4; ++s)
    if (4 * s + sub < n) Y[(4 * s + sub) * kXS + col] = y[s];
  __syncthreads();
  for (int e = tid; e < p.B * kGroups; e += kThreads) {
    const int i = e / kGroups, d = e % kGroups * 4;
    float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < n) w = *reinterpret_cast<const float4*>(Y + i * kXS + d);
    T* o = out + (size_t)i * p.Hv * DV + d;
    o[0] = from_f32<T>(p.scale * w.x);
    o[1] = from_f32<T>(p.scale * w.y);
    o[2] = from_f32<T>(p.scale * w.z);
    o[3] = from_f32<T>(p.scale * w.w);
  }
}

namespace {

template <typename T, int DK, int DV, int NODES>
cudaError_t launch_n(const GdrParams& p, cudaStream_t stream) {
  auto smem_for = [](int B) {
    const int rows = (B + 3) & ~3;
    return (int)sizeof(float) * (linear_state(DK, DV, rows) + rows * 2 * (DK + 4 + DV + 8));
  };
  cudaError_t e = cudaFuncSetAttribute(tree_linear_kernel<T, DK, DV, NODES>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       smem_for(NODES));
  if (e != cudaSuccess) return e;
  tree_linear_kernel<T, DK, DV, NODES>
      <<<(unsigned)((long)p.R * p.Hv), kParts * DV, smem_for(p.B), stream>>>(p);
  note_launches(1);
  return cudaGetLastError();
}

// Trees of at most 16 nodes take the kernel whose fewer registers let more CTAs run
// at once: 64 requests x 16 nodes x 32 heads, 64 x 64 bf16 46.8 -> 39.0 us, 128 x 128
// fp32 177 -> 124 us.
template <typename T, int DK, int DV>
cudaError_t launch_t(const GdrParams& p, cudaStream_t stream) {
  return p.B <= 16 ? launch_n<T, DK, DV, 16>(p, stream) : launch_n<T, DK, DV, kMaxNodes>(p, stream);
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
