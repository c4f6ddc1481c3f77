// State commit of an accepted path of a drafted tree, exact fp32 recurrence:
//     S <- alpha_t S,  delta_t = beta_t (v_t - S^T k_t),  S <- S + k_t delta_t^T
// for the path's tokens t in order (Eq. per-step-fwd), from the source slot's
// state into the destination slot.
//
// The rule acts on the state from the left, so its columns evolve on their
// own: a CTA takes 64 columns of one (request, value head).  A thread keeps 4
// columns x dk/8 rows in registers as fp32 pairs (packed f32x2 arithmetic);
// the 8 row groups of a column sit in one warp and meet in three shuffles.
// Bound by the state's bytes at serving path lengths (a round accepts a few
// tokens): the state moves once each way in 16-byte pieces, all of a thread's
// loads in flight together with the path's keys and values (two round trips to
// memory before the first step), and several CTAs per SM overlap one's loads
// with another's steps.  64 requests x 32 heads of 128 x 128, paths of 1 to 8:
// 50 us, 5.4 TB/s; one fp32 path of 33: 7.5 us, its steps one after another.
#include "common.cuh"
#include "kernels.h"
#include "tree.cuh"

namespace flare {

namespace {
constexpr int kCommitCols = 64;                   // state columns per CTA
constexpr int kCommitThreads = 2 * kCommitCols;   // a warp covers 16 columns
}  // namespace

template <typename T, int DK, int DV>
__global__ void __launch_bounds__(kCommitThreads, 4) tree_commit_kernel(GdrParams p) {
  constexpr int kR = DK / 8;  // state rows per thread
  constexpr int kSplit = DV / kCommitCols;
  extern __shared__ __align__(16) float sm[];
  __shared__ float2 gate_s[kMaxNodes];  // {alpha, beta}
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int item = blockIdx.x / kSplit, part = blockIdx.x % kSplit;
  const int r = item / p.Hv, j = item % p.Hv, h = j / (p.Hv / p.Hk);
  const int rg = lane >> 2;                     // row group: rows rg*kR ..
  const int c = warp * 16 + (lane & 3) * 4;     // this thread's columns within the CTA's
  const int src = p.state_slot[r], dst = p.dst_slot[r], n = p.accept_len[r];
  // rows of the path in the same round trip, before their number is known: a
  // thread's 16-byte pieces of the keys belong to steps tk, tk + kStepK, ..
  constexpr int kE = 16 / sizeof(T);
  constexpr int kPk = DK / kE, kStepK = kCommitThreads / kPk;            // key pieces, rows a pass
  constexpr int kPv = kCommitCols / kE, kStepV = kCommitThreads / kPv;   // value pieces
  const int tk = tid / kPk, tv = tid / kPv;
  const int32_t* path = p.path + (size_t)r * p.B;
  const int row_k = tk < p.B ? path[tk] : 0, row_v = tv < p.B ? path[tv] : 0;
  const int row_g = tid < p.B ? path[tid] : 0;
  // The state of the item a CTA per SM further on, into L2 while this one's steps
  // run: that CTA starts within a quarter of the resident ones' time (64 requests,
  // paths of 1 to 8: 51.6 us without, 49.8 at 152 CTAs' distance, 50.5 at 304, 52.2
  // at 608).
  if (tid == 0 && part == 0 && blockIdx.x + kNumSMs < gridDim.x) {
    const int x = (blockIdx.x + kNumSMs) / kSplit, slot = p.state_slot[x / p.Hv];
    const bool rests = p.accept_len[x / p.Hv] == 0 && p.dst_slot[x / p.Hv] == slot;
    if (slot >= 0 && slot < p.nslots && !rests)
      asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(
                       p.state_pool + ((size_t)slot * p.Hv + x % p.Hv) * DK * DV),
                   "r"(DK * DV * 4)
                   : "memory");
  }
  int bad = 0;
  if (src < 0 || src >= p.nslots || dst < 0 || dst >= p.nslots) bad |= FLARE_DEV_BAD_SLOT;
  if (n < 0 || n > p.B) bad |= FLARE_DEV_BAD_ACCEPT_LEN;
  if (bad) {
    if (tid == 0) flag(p.dev_status, bad);
    return;
  }
  if (n == 0 && src == dst) return;
  const size_t at = ((size_t)j * DK + rg * kR) * DV + part * kCommitCols + c;
  const size_t head = (size_t)p.Hv * DK * DV;
  const float* Sg = p.state_pool + src * head + at;
  uint64_t s[kR][2];  // S[rg*kR + m][columns c, c+1 | c+2, c+3]
#pragma unroll
  for (int m = 0; m < kR; ++m) {
    const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(Sg + (size_t)m * DV);
    s[m][0] = x.x;
    s[m][1] = x.y;
  }
  // the path's gates, keys and this CTA's value columns, as fp32
  float* Ks = sm;            // [n][DK]
  float* Vs = Ks + n * DK;   // [n][kCommitCols]
  const T* k = static_cast<const T*>(p.k) + ((size_t)r * p.B * p.Hk + h) * DK + tid % kPk * kE;
  const T* v = static_cast<const T*>(p.v) + ((size_t)r * p.B * p.Hv + j) * DV +
               part * kCommitCols + tid % kPv * kE;
  auto piece = [&](const T* x, int row, size_t stride, float* out) {
    if (row < 0 || row >= p.B) {
      bad = 1;
      return;
    }
    const uint4 w = *reinterpret_cast<const uint4*>(x + (size_t)row * stride);
    const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int i = 0; i < kE; ++i) out[i] = to_f32(e[i]);
  };
  for (int t = tk; t < n; t += kStepK)
    piece(k, t == tk ? row_k : path[t], (size_t)p.Hk * DK, Ks + t * DK + tid % kPk * kE);
  for (int t = tv; t < n; t += kStepV)
    piece(v, t == tv ? row_v : path[t], (size_t)p.Hv * DV, Vs + t * kCommitCols + tid % kPv * kE);
  if (tid < n && row_g >= 0 && row_g < p.B) {
    const size_t g = ((size_t)r * p.B + row_g) * p.Hv + j;
    gate_s[tid] = make_float2(expf(p.log_decay[g]), p.beta[g]);
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) flag(p.dev_status, FLARE_DEV_BAD_TREE);
    return;
  }
#pragma unroll 1
  for (int t = 0; t < n; ++t) {
    float kv[kR];
#pragma unroll
    for (int m = 0; m < kR; m += 4) {
      const float4 x = *reinterpret_cast<const float4*>(Ks + t * DK + rg * kR + m);
      kv[m] = x.x;
      kv[m + 1] = x.y;
      kv[m + 2] = x.z;
      kv[m + 3] = x.w;
    }
    const float2 gate = gate_s[t];
    const uint64_t a2 = f2_dup(gate.x);
    uint64_t d01[2] = {0, 0}, d23[2] = {0, 0};  // two partial sums: four independent chains
#pragma unroll
    for (int m = 0; m < kR; ++m) {
      const uint64_t k2 = f2_dup(kv[m]);
      d01[m & 1] = f2_fma(s[m][0], k2, d01[m & 1]);
      d23[m & 1] = f2_fma(s[m][1], k2, d23[m & 1]);
    }
    float4 d;
    f2_split(f2_add(d01[0], d01[1]), d.x, d.y);
    f2_split(f2_add(d23[0], d23[1]), d.z, d.w);
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      d.x += __shfl_xor_sync(0xffffffffu, d.x, o);
      d.y += __shfl_xor_sync(0xffffffffu, d.y, o);
      d.z += __shfl_xor_sync(0xffffffffu, d.z, o);
      d.w += __shfl_xor_sync(0xffffffffu, d.w, o);
    }
    const float4 x = *reinterpret_cast<const float4*>(Vs + t * kCommitCols + c);
    const uint64_t w01 = f2(gate.y * (x.x - gate.x * d.x), gate.y * (x.y - gate.x * d.y));
    const uint64_t w23 = f2(gate.y * (x.z - gate.x * d.z), gate.y * (x.w - gate.x * d.w));
#pragma unroll
    for (int m = 0; m < kR; ++m) {
      const uint64_t k2 = f2_dup(kv[m]);
      s[m][0] = f2_fma(k2, w01, f2_mul(a2, s[m][0]));
      s[m][1] = f2_fma(k2, w23, f2_mul(a2, s[m][1]));
    }
  }
  float* Dg = p.state_pool + dst * head + at;
#pragma unroll
  for (int m = 0; m < kR; ++m)
    *reinterpret_cast<ulonglong2*>(Dg + (size_t)m * DV) = make_ulonglong2(s[m][0], s[m][1]);
}

namespace {

template <typename T, int DK, int DV>
cudaError_t launch_t(const GdrParams& p, cudaStream_t stream) {
  auto smem_for = [](int B) { return (int)sizeof(float) * B * (DK + kCommitCols); };
  cudaError_t e = cudaFuncSetAttribute(tree_commit_kernel<T, DK, DV>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       smem_for(kMaxNodes));
  if (e != cudaSuccess) return e;
  const long long ctas = (long long)p.R * p.Hv * (DV / kCommitCols);
  if (ctas > INT32_MAX) return cudaErrorInvalidValue;
  tree_commit_kernel<T, DK, DV>
      <<<(unsigned)ctas, kCommitThreads, smem_for(p.B), stream>>>(p);
  note_launches(1);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_d(const GdrParams& p, cudaStream_t stream) {
  if (p.dk == 128 && p.dv == 128) return launch_t<T, 128, 128>(p, stream);
  if (p.dk == 128 && p.dv == 64) return launch_t<T, 128, 64>(p, stream);
  if (p.dk == 64 && p.dv == 128) return launch_t<T, 64, 128>(p, stream);
  if (p.dk == 64 && p.dv == 64) return launch_t<T, 64, 64>(p, stream);
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_tree_commit(const GdrParams& p, bool bf16, cudaStream_t stream) {
  if (p.R == 0) return cudaSuccess;
  return bf16 ? launch_d<__nv_bfloat16>(p, stream) : launch_d<float>(p, stream);
}

}  // namespace flare
