// Verification of drafted trees against the target's distributions.
//
//   tree_rows_kernel  log-sum-exp (and argmax) of every row that has children,
//                     in one pass over the logits: CTAs (chunk, row) leave a
//                     partial {max, sum, argmax} each
//   tree_walk_kernel  a cluster per request joins the partials, writes the
//                     drafted nodes' log-probabilities, walks the tree and
//                     draws the next token
//
// With siblings drawn independently from q, a rejection replaces the target by
// the normalised positive part of (target - q).  Iterating that telescopes:
// after j rejections the unnormalised residual is max(p - c_j q, 0) with
// c_0 = 0, c_{j+1} = c_j + m_j, m_j its mass (m_0 = 1), so no residual is
// stored, and a mass is only summed when another sibling is still to be tried.
// With fixed drafts the residual is p without the rejected tokens: their p comes
// off the mass, which is summed anew when little of it is left.
// The next token is the argmax of w / noise (noise ~ Exp(1) samples w).
//
// Bound by the logits' bytes on many rows and by latency on few.  The walk
// itself needs a dozen numbers per node, gathered by a thread each before it
// starts; what is long in it, a pass over one row, is cut over the cluster's
// CTAs, which all take the same decisions from the same numbers and exchange
// sums and maxima through distributed shared memory, in rank order.
//
// 64 trees of 16 nodes over 32000 tokens: 22.1 us sampled, half of it the row
// statistics (44 MB, 4 TB/s) and half the walk, which reads 18 MB more in two to
// four dependent passes per request; 23.2 us with fixed drafts, 18.7 greedy.  One
// greedy tree of 9 over 50257: 7.6 us.
//
// Logits enter by their differences alone (to a row's maximum, or to the best
// candidate so far): their products with the scale may overflow, at a type's lowest
// value, or leave no digits for a difference, at a low temperature.
#include "common.cuh"
#include "kernels.h"
#include "pdl.cuh"
#include "tc.cuh"
#include "tree.cuh"

namespace flare {

namespace {

constexpr int kRowThreads = 128;
constexpr int kWalkThreads = 512;
constexpr int kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;
// Fixed drafts: the part of a summed mass down to which differences from it are
// taken.  They are off by a few 2^-24 of that mass, so the rest by 2^-14 at most.
constexpr float kResum = 1.f / 256;

// The better of two (value, index) candidates: the greater value, the lower
// index among equals.
__device__ __forceinline__ void take_best(float& v, int& i, float v2, int i2) {
  if (v2 > v || (v2 == v && i2 < i)) {
    v = v2;
    i = i2;
  }
}

// The temperature as a factor on differences of logits, for powers of two.
__device__ __forceinline__ float log2_scale(float inv_temp) {
  return fminf(inv_temp * kLog2e, 3.402823466e38f);
}

// The same in a race of candidates of value 2^(scale v) / 2^e: by the difference of
// two, which keeps its digits where the products with the scale would lose them (a
// low temperature) or overflow (logits at the end of the type's range).
__device__ __forceinline__ void take_race(float& v, float& e, int& i, float v2, float e2, int i2,
                                          float scale) {
  const float d = fmaf(v2 - v, scale, e - e2);
  if (d > 0.f || (d == 0.f && i2 < i)) {
    v = v2;
    e = e2;
    i = i2;
  }
}

__device__ __forceinline__ void warp_race(float& v, float& e, int& i, float scale) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float v2 = __shfl_xor_sync(0xffffffffu, v, o);
    const float e2 = __shfl_xor_sync(0xffffffffu, e, o);
    const int i2 = __shfl_xor_sync(0xffffffffu, i, o);
    take_race(v, e, i, v2, e2, i2, scale);
  }
}

__device__ __forceinline__ void warp_best(float& v, int& i) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float v2 = __shfl_xor_sync(0xffffffffu, v, o);
    const int i2 = __shfl_xor_sync(0xffffffffu, i, o);
    take_best(v, i, v2, i2);
  }
}

// {max, sum of 2^(scale (x - max)), argmax} of a row from its parts on a warp's
// lanes: the maximum first, then one rescaling per part.  Maxima are the logits
// themselves: times the scale, neighbouring floats can round to one value.
__device__ __forceinline__ float4 warp_stats(float4 st, float scale) {
  float m = st.x;
  int best = (int)st.z;
  warp_best(m, best);
  float s = st.x == -INFINITY ? st.y : st.y * tc::ex2(scale * (st.x - m));  // a NaN sum stays one
  s = warp_sum(s);
  return make_float4(m, s, (float)best, 0.f);
}

}  // namespace

// A chunk of a row: 16-byte loads over its aligned middle, eight of them in
// flight per thread, and single elements at both ends (a row may start at any
// element).  The running maximum moves once per batch, not per element.
template <typename T, bool GREEDY>
__global__ void __launch_bounds__(kRowThreads) tree_rows_kernel(TreeVerifyParams p) {
  constexpr int kE = 16 / sizeof(T), kIn = 8;
  __shared__ float4 red[kRowThreads / 32];
  pdl_launch_next();
  const int row = blockIdx.y, r = row / p.N, i = row - r * p.N, tid = threadIdx.x;
  {  // rows without children are read only where a walk ends
    const int32_t* par = p.parent + (size_t)r * p.N;
    const int lane = tid & 31;
    // both in one round trip, unused nodes' entries (any value) masked after it
    const int n = p.node_len[r];
    const int p0 = lane < p.N ? par[lane] : -1, p1 = lane + 32 < p.N ? par[lane + 32] : -1;
    const bool kid = (lane < n && p0 == i) || (lane + 32 < n && p1 == i);
    // the same in every warp; a wrong length is flagged by the walk
    if (n > p.N || i >= n || !__any_sync(0xffffffffu, kid)) return;
  }
  const int lo = blockIdx.x * p.chunk, hi = min(p.V, lo + p.chunk);
  const T* x = static_cast<const T*>(p.logits) + (size_t)row * p.V;
  const float scale = log2_scale(p.inv_temp);
  float m = -INFINITY, s = 0.f;  // maximum of the raw logits, sum of 2^(scale (x - m))
  int best = p.V;
  auto one = [&](int at) {
    const float v = to_f32(x[at]);
    if (v > m) {
      s *= tc::ex2(scale * (m - v));
      m = v;
      best = at;
    } else if (GREEDY && v == m) {
      best = min(best, at);
    }
    if (v != -INFINITY) s += tc::ex2(scale * (v - m));  // a NaN makes the sum one
  };
  const int skew = (int)(((uintptr_t)(x + lo) & 15u) / sizeof(T));
  const int a = min(hi, skew ? lo + kE - skew : lo);  // first aligned element
  const int nv = (hi - a) / kE, tail = a + nv * kE;
  if (tid < a - lo) one(lo + tid);
  const uint4* vec = reinterpret_cast<const uint4*>(x + a);
  for (int i0 = tid; i0 < nv; i0 += kIn * kRowThreads) {
    uint4 w[kIn];
#pragma unroll
    for (int u = 0; u < kIn; ++u)
      if (i0 + u * kRowThreads < nv) w[u] = __ldcs(vec + i0 + u * kRowThreads);
#pragma unroll
    for (int u = 0; u < kIn; ++u) {
      if (i0 + u * kRowThreads >= nv) continue;
      float v[kE];
      if constexpr (sizeof(T) == 2) {
        const uint32_t h[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[2 * k] = __uint_as_float(h[k] << 16);
          v[2 * k + 1] = __uint_as_float(h[k] & 0xffff0000u);
        }
      } else {
        v[0] = __uint_as_float(w[u].x);
        v[1] = __uint_as_float(w[u].y);
        v[2] = __uint_as_float(w[u].z);
        v[3] = __uint_as_float(w[u].w);
      }
      float bm = v[0];
#pragma unroll
      for (int k = 1; k < kE; ++k) bm = fmaxf(bm, v[k]);
      if (bm > m) {
        s *= tc::ex2(scale * (m - bm));
        m = bm;
        if constexpr (GREEDY) {
          const int base = a + (i0 + u * kRowThreads) * kE;
#pragma unroll
          for (int k = kE - 1; k >= 0; --k)
            if (v[k] == bm) best = base + k;
        }
      } else if (GREEDY && bm == m) {  // equal to an element of a scalar end further right
        const int base = a + (i0 + u * kRowThreads) * kE;
#pragma unroll
        for (int k = kE - 1; k >= 0; --k)
          if (v[k] == bm) best = min(best, base + k);
      }
      // differences first: the lowest finite logit times the scale overflows
      const uint64_t neg = f2_dup(m == -INFINITY ? 0.f : -m), scale2 = f2_dup(scale);
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int k = 0; k < kE; k += 2) {
        float d0, d1;
        f2_split(f2_mul(scale2, f2_add(f2(v[k], v[k + 1]), neg)), d0, d1);
        s0 += tc::ex2(d0);
        s1 += tc::ex2(d1);
      }
      s += s0 + s1;
    }
  }
  if (tid < hi - tail) one(tail + tid);
  float4 st = warp_stats(make_float4(m, s, (float)best, 0.f), scale);
  if ((tid & 31) == 0) red[tid >> 5] = st;
  __syncthreads();
  if (tid < 32) {
    st = warp_stats(tid < kRowThreads / 32 ? red[tid]
                                           : make_float4(-INFINITY, 0.f, (float)p.V, 0.f),
                    scale);
    if (tid == 0) p.stats[(size_t)row * p.n_chunks + blockIdx.x] = st;
  }
}

namespace {

// p - c q of two tokens, p = 2^(scale (x - mx) - ls2).
__device__ __forceinline__ void residual(float x0, float x1, float q0, float q1, float mx,
                                         float ls2, float scale, float c, float& w0, float& w1) {
  float p0, p1;
  f2_split(f2_fma(f2_add(f2(x0, x1), f2_dup(-mx)), f2_dup(scale), f2_dup(-ls2)), p0, p1);
  f2_split(f2_fma(f2(q0, q1), f2_dup(-c), f2(tc::ex2(p0), tc::ex2(p1))), w0, w1);
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t x;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(x));
  return x;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t x;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(x));
  return x;
}
// Every thread of the cluster; orders shared-memory writes before remote reads.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A 32-bit word of shared memory of the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t cluster_word(const void* mine, uint32_t rank) {
  uint32_t at, x;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
               : "=r"(at)
               : "r"(tc::smem_u32(mine)), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}

struct WalkShared {
  int par[kMaxNodes], tok[kMaxNodes], line[kMaxNodes], best_of[kMaxNodes], gone[kMaxNodes];
  unsigned long long kids[kMaxNodes];
  float uni[kMaxNodes], logp[kMaxNodes], q[kMaxNodes], prob[kMaxNodes];
  float mx[kMaxNodes], ls2[kMaxNodes];  // a row's maximum, log2 of its sum
  float red_v[kWalkThreads / 32], red_e[kWalkThreads / 32];
  int red_i[kWalkThreads / 32];
  int tree_ok;
  // the walk: the node it stands at, its path, the residual there
  int cur, len, more, n_gone;
  unsigned long long left;  // children still to be tried
  float c, m, summed;       // summed: the mass when it was last a sum
  // this CTA's share of a pass over a row, in two buffers: a CTA is at most
  // one pass ahead of another that still reads its last share
  float part_v[2], part_e[2];
  int part_i[2], part_odd[2];
};

}  // namespace

template <typename T>
__global__ void __launch_bounds__(kWalkThreads) tree_walk_kernel(TreeVerifyParams p) {
  constexpr int kWarps = kWalkThreads / 32;
  __shared__ WalkShared sh;
  const uint32_t rank = cluster_rank(), ranks = cluster_size();
  const int r = blockIdx.x / ranks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = p.node_len[r];
  // every CTA of a cluster comes to the same answer at each of these exits
  if (n < 0 || n > p.N) {
    if (tid == 0 && rank == 0) flag(p.dev_status, FLARE_DEV_BAD_TREE);
    pdl_wait();
    return;
  }
  const bool sample = !p.greedy;
  if (tid < 32) {
    int p0, p1;
    const bool ok = warp_load_tree(p.parent + (size_t)r * p.N, n, p0, p1);
    sh.par[tid] = p0;
    sh.par[tid + 32] = p1;
    sh.kids[tid] = sh.kids[tid + 32] = 0ull;
    __syncwarp();
    if (ok) {
      if (p0 >= 0) atomicOr(&sh.kids[p0], 1ull << tid);
      if (p1 >= 0) atomicOr(&sh.kids[p1], 1ull << (tid + 32));
    }
    if (tid == 0) sh.tree_ok = ok;
  } else if (tid >= 64 && tid < 64 + kMaxNodes) {
    const int i = tid - 64;
    const bool drafted = i > 0 && i < n;
    sh.tok[i] = drafted ? p.token[(size_t)r * p.N + i] : 0;
    sh.uni[i] = drafted && sample ? p.uniform[(size_t)r * p.N + i] : 0.f;
  }
  __syncthreads();
  int bad = sh.tree_ok ? 0 : FLARE_DEV_BAD_TREE;
  if (tid < kMaxNodes && (sh.tok[tid] < 0 || sh.tok[tid] >= p.V)) bad = FLARE_DEV_BAD_TREE;
  if (__syncthreads_or(bad)) {
    if (tid == 0 && rank == 0) flag(p.dev_status, FLARE_DEV_BAD_TREE);
    pdl_wait();
    return;
  }
  if (n == 0) {
    if (rank == 0 && tid < p.N) {
      p.path[(size_t)r * p.N + tid] = -1;
      p.node_logp[(size_t)r * p.N + tid] = 0.f;
    }
    if (rank == 0 && tid == 0) {
      p.path_len[r] = 0;
      p.next_token[r] = -1;
    }
    pdl_wait();
    return;
  }
  const T* rows = static_cast<const T*>(p.logits) + (size_t)r * p.N * p.V;
  const float scale = log2_scale(p.inv_temp);
  const float* drafts =
      sample && p.draft_probs ? p.draft_probs + (size_t)r * p.N * p.V : nullptr;
  float x_tok = 0.f;  // the drafted token's logit, and its probability for the drafter
  if (tid > 0 && tid < n) {
    const size_t at = (size_t)sh.par[tid] * p.V + sh.tok[tid];
    x_tok = to_f32(rows[at]);
    sh.q[tid] = drafts ? drafts[at] : 1.f;
  }
  const int lo = (int)((long long)p.V * rank / ranks), hi = (int)((long long)p.V * (rank + 1) / ranks);
  pdl_wait();  // the row statistics
  // a warp per row with children: its log-sum-exp and argmax
  for (int i = warp; i < n; i += kWarps) {
    if (!sh.kids[i]) continue;
    float4 st = make_float4(-INFINITY, 0.f, (float)p.V, 0.f);
    for (int c0 = 0; c0 < p.n_chunks; c0 += 31) {  // 31 parts and what came before
      if (lane > 0)
        st = c0 + lane - 1 < p.n_chunks
                 ? p.stats[((size_t)r * p.N + i) * p.n_chunks + c0 + lane - 1]
                 : make_float4(-INFINITY, 0.f, (float)p.V, 0.f);
      st = warp_stats(st, scale);
    }
    if (lane == 0) {
      sh.mx[i] = st.x;
      sh.ls2[i] = log2f(st.y);
      sh.best_of[i] = (int)st.z;
      if (!(fabsf(st.x) < INFINITY && st.y < INFINITY)) bad = FLARE_DEV_BAD_LOGITS;
    }
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0 && rank == 0) flag(p.dev_status, FLARE_DEV_BAD_LOGITS);
    return;
  }
  if (tid < kMaxNodes) {
    const bool drafted = tid > 0 && tid < n;
    const int at = drafted ? sh.par[tid] : 0;
    const float d = x_tok - sh.mx[at], ls2 = sh.ls2[at];
    sh.logp[tid] = drafted ? fmaf(d, p.inv_temp, ls2 * -0.6931471805599453f) : 0.f;
    sh.prob[tid] = drafted ? exp2f(fmaf(d, scale, -ls2)) : 0.f;
  }
  if (tid == 0) {
    sh.cur = 0;
    sh.len = 1;
    sh.line[0] = 0;
    sh.left = sh.kids[0];
    sh.c = 0.f;
    sh.m = sh.summed = 1.f;
    sh.n_gone = 0;
  }
  __syncthreads();

  // Calls f(x, ...) for this CTA's tokens of a row, kIn of a thread's loads in
  // flight: consecutive threads on consecutive tokens, whatever the alignment.
  constexpr int kIn = 8;
  int pass = 0;

  // The walk: thread 0 tries children until it needs a mass (then the cluster
  // sums it) or is done.
  while (true) {
    if (tid == 0) {
      int cur = sh.cur, len = sh.len, more = 0;
      unsigned long long left = sh.left;
      float c = sh.c, m = sh.m, summed = sh.summed;
      while (left) {
        const int i = __ffsll((long long)left) - 1;
        left &= left - 1;
        bool ok;
        if (!sample) {
          ok = sh.tok[i] == sh.best_of[cur];
        } else {
          const float px = sh.prob[i];
          if (drafts) {
            ok = sh.uni[i] * sh.q[i] * m < fmaxf(px - c * sh.q[i], 0.f);
            if (!ok) {
              c += m;
              if (left) {  // another sibling: the residual's mass is needed
                more = 1;
                break;
              }
            }
          } else {
            bool was = false;
            for (int e = 0; e < sh.n_gone; ++e) was = was || sh.gone[e] == sh.tok[i];
            ok = !was && sh.uni[i] * m < px;
            if (!ok && !was) {
              sh.gone[sh.n_gone++] = sh.tok[i];
              m = fmaxf(m - px, 0.f);
              if (left && m < kResum * summed) {
                more = 1;
                break;
              }
            }
          }
        }
        if (ok) {
          cur = i;
          sh.line[len++] = i;
          left = sh.kids[i];
          c = 0.f;
          m = summed = 1.f;
          sh.n_gone = 0;
        }
      }
      sh.cur = cur;
      sh.len = len;
      sh.left = left;
      sh.c = c;
      sh.m = m;
      sh.summed = summed;
      sh.more = more;
    }
    __syncthreads();
    if (!sh.more) break;
    const T* x = rows + (size_t)sh.cur * p.V;
    const float c = sh.c, mx = sh.mx[sh.cur], ls2 = sh.ls2[sh.cur];
    float sum = 0.f;
    if (drafts) {
      const float* q = drafts + (size_t)sh.cur * p.V;
      for (int t0 = lo + tid; t0 < hi; t0 += kIn * kWalkThreads) {
        float xv[kIn], qv[kIn];
#pragma unroll
        for (int u = 0; u < kIn; ++u) {
          const int t = t0 + u * kWalkThreads;
          xv[u] = t < hi ? to_f32(x[t]) : -INFINITY;
          qv[u] = t < hi ? q[t] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kIn; u += 2) {
          float w0, w1;
          residual(xv[u], xv[u + 1], qv[u], qv[u + 1], mx, ls2, scale, c, w0, w1);
          sum += fmaxf(w0, 0.f) + fmaxf(w1, 0.f);
        }
      }
    } else {
      const int ng = sh.n_gone;
#pragma unroll 1
      for (int t = lo + tid; t < hi; t += kWalkThreads) {
        bool in = true;
#pragma unroll 1
        for (int e = 0; e < ng; ++e) in = in && sh.gone[e] != t;
        if (in) sum += tc::ex2(fmaf(to_f32(x[t]) - mx, scale, -ls2));
      }
    }
    sum = warp_sum(sum);
    if (lane == 0) sh.red_v[warp] = sum;
    __syncthreads();
    if (warp == 0) {
      const float m = warp_sum(lane < kWarps ? sh.red_v[lane] : 0.f);
      if (lane == 0) sh.part_v[pass & 1] = m;
    }
    cluster_sync();
    if (warp == 0) {
      const float m = warp_sum(
          lane < (int)ranks ? __uint_as_float(cluster_word(&sh.part_v[pass & 1], lane)) : 0.f);
      if (lane == 0) sh.m = sh.summed = m;
    }
    ++pass;
    __syncthreads();
  }

  // The next token, from the last accepted node's row.
  const int cur = sh.cur;
  int next = 0, odd = 0;
  if (!sample && sh.kids[cur]) {
    next = sh.best_of[cur];
  } else {
    const T* x = rows + (size_t)cur * p.V;
    const float* noise = sample ? p.noise + (size_t)r * p.V : nullptr;
    float c = drafts ? sh.c : 0.f;
    int ng = sh.n_gone;
    while (true) {
      const float* q = c > 0.f ? drafts + (size_t)cur * p.V : nullptr;
      const float mx = q ? sh.mx[cur] : 0.f, ls2 = q ? sh.ls2[cur] : 0.f;
      const bool race = sample && !q;  // candidates as {logit, log2 noise}, else as values
      const float by = race ? scale : 1.f;
      float v0 = -INFINITY, e0 = 0.f, top = -INFINITY;  // top: a NaN once one was read
      int i0 = p.V;
      // tokens come in ascending order: the first of equals stays.  Quotients and
      // powers to 2 ulp, and w = p - c q to 2 ulp of p: only candidates that close to
      // equal can change places.
      auto take = [&](bool ok, float v, int t) {
        if (ok && v > v0) {
          v0 = v;
          i0 = t;
        }
      };
      for (int t0 = lo + tid; t0 < hi; t0 += kIn * kWalkThreads) {
        float xv[kIn], ev[kIn], qv[kIn];
#pragma unroll
        for (int u = 0; u < kIn; ++u) {
          const int t = t0 + u * kWalkThreads;
          xv[u] = t < hi ? to_f32(x[t]) : -INFINITY;
          ev[u] = noise && t < hi ? noise[t] : 1.f;
          qv[u] = q && t < hi ? q[t] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kIn; ++u)
          asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(xv[u]));
        if (!sample) {
#pragma unroll
          for (int u = 0; u < kIn; ++u) take(true, xv[u], t0 + u * kWalkThreads);
        } else if (q) {
#pragma unroll
          for (int u = 0; u < kIn; u += 2) {
            float w0, w1;
            residual(xv[u], xv[u + 1], qv[u], qv[u + 1], mx, ls2, scale, c, w0, w1);
            take(w0 > 0.f, __fdividef(w0, ev[u]), t0 + u * kWalkThreads);
            take(w1 > 0.f, __fdividef(w1, ev[u + 1]), t0 + (u + 1) * kWalkThreads);
          }
        } else {  // in logarithms, against the best so far: no normaliser is needed
#pragma unroll
          for (int u = 0; u < kIn; ++u) {
            const int t = t0 + u * kWalkThreads;
            bool in = true;
            for (int e = 0; e < ng; ++e) in = in && sh.gone[e] != t;
            const float e = log2f(ev[u]);
            if (in && fmaf(xv[u] - v0, scale, e0 - e) > 0.f) {
              v0 = xv[u];
              e0 = e;
              i0 = t;
            }
          }
        }
      }
      odd |= !(top < INFINITY);
      warp_race(v0, e0, i0, by);
      if (lane == 0) {
        sh.red_v[warp] = v0;
        sh.red_e[warp] = e0;
        sh.red_i[warp] = i0;
      }
      const int any_odd = __syncthreads_or(odd);
      if (warp == 0) {
        v0 = lane < kWarps ? sh.red_v[lane] : -INFINITY;
        e0 = lane < kWarps ? sh.red_e[lane] : 0.f;
        i0 = lane < kWarps ? sh.red_i[lane] : p.V;
        warp_race(v0, e0, i0, by);
        if (lane == 0) {
          sh.part_v[pass & 1] = v0;
          sh.part_e[pass & 1] = e0;
          sh.part_i[pass & 1] = i0;
          sh.part_odd[pass & 1] = any_odd;
        }
      }
      cluster_sync();
      if (warp == 0) {
        v0 = -INFINITY;
        e0 = 0.f;
        i0 = p.V;
        int o = 0;
        if (lane < (int)ranks) {
          v0 = __uint_as_float(cluster_word(&sh.part_v[pass & 1], lane));
          e0 = __uint_as_float(cluster_word(&sh.part_e[pass & 1], lane));
          i0 = (int)cluster_word(&sh.part_i[pass & 1], lane);
          o = (int)cluster_word(&sh.part_odd[pass & 1], lane);
        }
        warp_race(v0, e0, i0, by);
        o = __any_sync(0xffffffffu, o);
        if (lane == 0) {
          sh.red_i[0] = i0;
          sh.red_i[1] = o;
        }
      }
      ++pass;
      __syncthreads();
      next = sh.red_i[0];
      odd = sh.red_i[1];
      if (odd || next < p.V || (c == 0.f && ng == 0)) break;
      __syncthreads();
      c = 0.f;  // nothing left of the residual: the target itself
      ng = 0;
    }
    cluster_sync();  // nobody leaves while its share may still be read
    if (next >= p.V) odd = 1;
  }
  if (rank != 0) return;
  if (odd) {
    if (tid == 0) flag(p.dev_status, FLARE_DEV_BAD_LOGITS);
    return;
  }
  if (tid < p.N) {
    p.path[(size_t)r * p.N + tid] = tid < sh.len ? sh.line[tid] : -1;
    p.node_logp[(size_t)r * p.N + tid] = sh.logp[tid];
  }
  if (tid == 0) {
    p.path_len[r] = sh.len;
    p.next_token[r] = next;
  }
}

void plan_tree_verify(int R, int N, int V, int num_sms, int* chunk, int* n_chunks) {
  // enough chunks for a few CTAs per SM, each with 4 to 32 KiB of bf16 logits
  const long long want = 8LL * num_sms;
  const long long rows = (long long)R * N > 0 ? (long long)R * N : 1;
  long long per = (want + rows - 1) / rows;
  long long len = (V + per - 1) / per;
  if (len < 2048) len = 2048;
  if (len > 16384) len = 16384;
  len = (len + 7) / 8 * 8;
  *chunk = (int)len;
  *n_chunks = (int)((V + len - 1) / len);
}

namespace {
template <typename T>
cudaError_t launch_t(const TreeVerifyParams& p, cudaStream_t stream) {
  const bool rows = p.N > 1;  // a lone anchor has no row with children
  if (rows) {
    TreeVerifyParams b = p;
    const int step = 65535 / p.N;  // requests per launch: rows go along the grid's y
    for (int r0 = 0; r0 < p.R; r0 += step) {
      const int nr = p.R - r0 < step ? p.R - r0 : step;
      const size_t e = (size_t)r0 * p.N;
      b.logits = static_cast<const T*>(p.logits) + e * p.V;
      b.parent = p.parent + e;
      b.node_len = p.node_len + r0;
      b.stats = p.stats + e * p.n_chunks;
      const dim3 grid((unsigned)p.n_chunks, (unsigned)(nr * p.N));
      if (p.greedy) tree_rows_kernel<T, true><<<grid, kRowThreads, 0, stream>>>(b);
      else tree_rows_kernel<T, false><<<grid, kRowThreads, 0, stream>>>(b);
      note_launches(1);
      const cudaError_t err = cudaGetLastError();
      if (err != cudaSuccess) return err;
    }
  }
  // CTAs per request: more while a share keeps 2048 tokens and the batch does
  // not yet fill the GPU
  int cluster = 1;
  while (cluster < kMaxCluster && p.V / (2 * cluster) >= 2048 &&
         (long long)p.R * 2 * cluster <= 2LL * kNumSMs)
    cluster *= 2;
  const cudaError_t err =
      pdl_launch(tree_walk_kernel<T>, dim3((unsigned)p.R * cluster), kWalkThreads, 0, stream, rows,
                 cluster, p);
  note_launches(1);
  return err != cudaSuccess ? err : cudaGetLastError();
}
}  // namespace

cudaError_t launch_tree_verify(const TreeVerifyParams& p, bool bf16, cudaStream_t stream) {
  if (p.R == 0) return cudaSuccess;
  return bf16 ? launch_t<__nv_bfloat16>(p, stream) : launch_t<float>(p, stream);
}

}  // namespace flare
