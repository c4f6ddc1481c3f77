// Verification of drafted trees against the target's distributions.
//
//   tree_rows_kernel  log-sum-exp and argmax of every row that has children, in
//                     one pass over the logits: CTAs (chunk, row) leave a
//                     partial {max, sum, argmax} each
//   tree_walk_kernel  a CTA per request joins the partials, writes the drafted
//                     nodes' log-probabilities, walks the tree and draws the
//                     next token
//
// With siblings drawn independently from q, a rejection replaces the target by
// the normalised positive part of (target - q).  Iterating that telescopes:
// after j rejections the unnormalised residual is max(p - c_j q, 0) with
// c_0 = 0, c_{j+1} = c_j + m_j, m_j its mass (m_0 = 1), so no residual is
// stored, and a mass is only summed when another sibling is still to be tried.
// With fixed drafts the residual is p without the rejected tokens.
// The next token is the argmax of w / noise (noise ~ Exp(1) samples w).
#include "common.cuh"
#include "kernels.h"
#include "tree.cuh"

namespace flare {

namespace {

constexpr int kRowThreads = 256;
constexpr int kWalkThreads = 1024;
constexpr float kLog2e = 1.4426950408889634f;

// Calls f(x, value) for the elements [lo, hi) of a row that may start at any
// element: 16-byte loads over the aligned middle, kIn of them in flight per
// thread, single elements at both ends.
template <typename T, int THREADS, typename F>
__device__ __forceinline__ void for_row(const T* row, int lo, int hi, F&& f) {
  constexpr int kE = 16 / sizeof(T), kIn = 4;
  const int tid = threadIdx.x;
  const int skew = (int)(((uintptr_t)(row + lo) & 15u) / sizeof(T));
  const int a = min(hi, skew ? lo + kE - skew : lo);  // first aligned element
  const int nv = (hi - a) / kE;
  if (tid < a - lo) f(lo + tid, to_f32(row[lo + tid]));
  const int tail = a + nv * kE;
  if (tid < hi - tail) f(tail + tid, to_f32(row[tail + tid]));
  const uint4* v = reinterpret_cast<const uint4*>(row + a);
  for (int i0 = tid; i0 < nv; i0 += kIn * THREADS) {
    uint4 x[kIn];
#pragma unroll
    for (int u = 0; u < kIn; ++u)
      if (i0 + u * THREADS < nv) x[u] = v[i0 + u * THREADS];
#pragma unroll
    for (int u = 0; u < kIn; ++u) {
      if (i0 + u * THREADS < nv) {
        const T* e = reinterpret_cast<const T*>(&x[u]);
        const int base = a + (i0 + u * THREADS) * kE;
#pragma unroll
        for (int k = 0; k < kE; ++k) f(base + k, to_f32(e[k]));
      }
    }
  }
}

// The better of two (value, index) candidates: the greater value, the lower
// index among equals.
__device__ __forceinline__ void take_best(float& v, int& i, float v2, int i2) {
  if (v2 > v || (v2 == v && i2 < i)) {
    v = v2;
    i = i2;
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

// {max, sum of exp(x - max), argmax} of two disjoint parts of a row
__device__ __forceinline__ float4 join_stats(float4 a, float4 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return make_float4(m, a.y + b.y, fminf(a.z, b.z), 0.f);
  const float s = a.y * expf(a.x - m) + b.y * expf(b.x - m);
  return make_float4(m, s, a.x > b.x ? a.z : b.x > a.x ? b.z : fminf(a.z, b.z), 0.f);
}

}  // namespace

template <typename T>
__global__ void __launch_bounds__(kRowThreads) tree_rows_kernel(TreeVerifyParams p) {
  __shared__ float4 red[kRowThreads / 32];
  __shared__ int inner;
  const int row = blockIdx.y, r = row / p.N, i = row - r * p.N, tid = threadIdx.x;
  const int n = p.node_len[r];
  if (n < 0 || n > p.N || i >= n) return;  // a wrong length is flagged by the walk
  if (tid < 32) {
    const int32_t* par = p.parent + (size_t)r * p.N;
    const bool kid = (tid < n && par[tid] == i) || (tid + 32 < n && par[tid + 32] == i);
    const bool any = __any_sync(0xffffffffu, kid);
    if (tid == 0) inner = any;
  }
  __syncthreads();
  if (!inner) return;
  const int lo = blockIdx.x * p.chunk, hi = min(p.V, lo + p.chunk);
  const T* x = static_cast<const T*>(p.logits) + (size_t)row * p.V;
  const float scale = p.inv_temp * kLog2e;
  // running maximum of the raw logits, moved lazily: sum of 2^(scale (x - m))
  float m = -INFINITY, s = 0.f;
  int best = p.V;
  for_row<T, kRowThreads>(x, lo, hi, [&](int at, float v) {
    if (v > m) {
      s *= exp2f(scale * (m - v));
      m = v;
      best = at;
    } else if (v == m && at < best) {
      best = at;
    }
    if (v != -INFINITY) s += exp2f(scale * (v - m));  // a NaN makes the sum one
  });
  float4 st = make_float4(m * p.inv_temp, s, (float)best, 0.f);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    float4 y;
    y.x = __shfl_xor_sync(0xffffffffu, st.x, o);
    y.y = __shfl_xor_sync(0xffffffffu, st.y, o);
    y.z = __shfl_xor_sync(0xffffffffu, st.z, o);
    st = join_stats(st, y);
  }
  if ((tid & 31) == 0) red[tid >> 5] = st;
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int w = 1; w < kRowThreads / 32; ++w) st = join_stats(st, red[w]);
    p.stats[(size_t)row * p.n_chunks + blockIdx.x] = st;
  }
}

template <typename T>
__global__ void __launch_bounds__(kWalkThreads) tree_walk_kernel(TreeVerifyParams p) {
  constexpr int kWarps = kWalkThreads / 32;
  __shared__ int par[kMaxNodes], tok[kMaxNodes], line[kMaxNodes], best_of[kMaxNodes];
  __shared__ float uni[kMaxNodes], logp[kMaxNodes], lse[kMaxNodes];
  __shared__ float red_v[kWarps];
  __shared__ int red_i[kWarps];
  __shared__ int tree_ok, inner_lo, inner_hi;
  __shared__ int s_cur, s_len, s_next, s_more, s_gone;
  __shared__ int gone[kMaxNodes];
  __shared__ float s_c, s_m;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = p.node_len[r];
  if (n < 0 || n > p.N) {
    if (tid == 0) flag(p.dev_status, FLARE_DEV_BAD_TREE);
    return;
  }
  const bool sample = !p.greedy;
  if (tid < 32) {
    int p0, p1;
    const bool ok = warp_load_tree(p.parent + (size_t)r * p.N, n, p0, p1);
    par[tid] = p0;
    par[tid + 32] = p1;
    if (tid == 0) {
      tree_ok = ok;
      inner_lo = inner_hi = 0;
      s_cur = 0;
      s_len = 1;
      s_c = 0.f;
      s_m = 1.f;
      s_gone = 0;
      s_next = 1;
      line[0] = 0;
    }
  }
  __syncthreads();
  int bad = tree_ok ? 0 : FLARE_DEV_BAD_TREE;
  if (tid < kMaxNodes && tid > 0 && tid < n) {
    const int x = p.token[(size_t)r * p.N + tid];
    tok[tid] = x;
    if (x < 0 || x >= p.V) bad |= FLARE_DEV_BAD_TREE;
    if (sample) uni[tid] = p.uniform[(size_t)r * p.N + tid];
  }
  if (__syncthreads_or(bad)) {
    if (bad && (tid == 0 || tree_ok)) flag(p.dev_status, bad);
    return;
  }
  if (n == 0) {
    if (tid < p.N) {
      p.path[(size_t)r * p.N + tid] = -1;
      p.node_logp[(size_t)r * p.N + tid] = 0.f;
    }
    if (tid == 0) {
      p.path_len[r] = 0;
      p.next_token[r] = -1;
    }
    return;
  }
  if (tid > 0 && tid < n) {  // which nodes have children
    const int a = par[tid];
    atomicOr(a < 32 ? &inner_lo : &inner_hi, 1 << (a & 31));
  }
  __syncthreads();
  auto is_inner = [&](int i) { return ((i < 32 ? inner_lo : inner_hi) >> (i & 31)) & 1; };
  // a warp per row with children: its log-sum-exp and argmax
  for (int i = warp; i < n; i += kWarps) {
    if (!is_inner(i)) continue;
    float4 st = make_float4(-INFINITY, 0.f, (float)p.V, 0.f);
    for (int c = lane; c < p.n_chunks; c += 32)
      st = join_stats(st, p.stats[((size_t)r * p.N + i) * p.n_chunks + c]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      float4 y;
      y.x = __shfl_xor_sync(0xffffffffu, st.x, o);
      y.y = __shfl_xor_sync(0xffffffffu, st.y, o);
      y.z = __shfl_xor_sync(0xffffffffu, st.z, o);
      st = join_stats(st, y);
    }
    if (lane == 0) {
      lse[i] = st.x + logf(st.y);
      best_of[i] = (int)st.z;
      if (!(fabsf(lse[i]) < INFINITY)) bad = FLARE_DEV_BAD_LOGITS;
    }
  }
  if (__syncthreads_or(bad)) {
    if (bad) flag(p.dev_status, bad);
    return;
  }
  const T* rows = static_cast<const T*>(p.logits) + (size_t)r * p.N * p.V;
  const float* drafts =
      sample && p.draft_probs ? p.draft_probs + (size_t)r * p.N * p.V : nullptr;
  if (tid < n)
    logp[tid] = tid == 0 ? 0.f
                         : to_f32(rows[(size_t)par[tid] * p.V + tok[tid]]) * p.inv_temp - lse[par[tid]];
  __syncthreads();

  // The walk: thread 0 tries siblings until it needs a mass (then the CTA sums
  // it) or is done.
  while (true) {
    if (tid == 0) {
      int cur = s_cur, len = s_len, more = 0, i = s_next;
      float c = s_c, m = s_m;
      for (; i < n; ++i) {
        if (par[i] != cur) continue;
        bool ok;
        if (!sample) {
          ok = tok[i] == best_of[cur];
        } else {
          const float px = expf(logp[i]);
          if (drafts) {
            const float q = drafts[(size_t)cur * p.V + tok[i]];
            ok = uni[i] * q * m < fmaxf(px - c * q, 0.f);
            if (!ok) {
              c += m;
              bool another = false;
              for (int e = i + 1; e < n; ++e) another = another || par[e] == cur;
              if (another) {  // its mass is needed
                more = 1;
                ++i;
                break;
              }
            }
          } else {
            bool was = false;
            for (int e = 0; e < s_gone; ++e) was = was || gone[e] == tok[i];
            ok = !was && uni[i] * m < px;
            if (!ok && !was) {
              gone[s_gone++] = tok[i];
              m = fmaxf(m - px, 0.f);
            }
          }
        }
        if (ok) {
          cur = i;
          line[len++] = i;
          c = 0.f;
          m = 1.f;
          s_gone = 0;
        }
      }
      s_cur = cur;
      s_len = len;
      s_next = i;
      s_c = c;
      s_m = m;
      s_more = more;
    }
    __syncthreads();
    if (!s_more) break;
    const T* x = rows + (size_t)s_cur * p.V;
    const float* q = drafts + (size_t)s_cur * p.V;
    const float c = s_c, shift = lse[s_cur] * kLog2e, scale = p.inv_temp * kLog2e;
    float sum = 0.f;
    for_row<T, kWalkThreads>(x, 0, p.V, [&](int at, float v) {
      sum += fmaxf(exp2f(v * scale - shift) - c * q[at], 0.f);
    });
    sum = warp_sum(sum);
    if (lane == 0) red_v[warp] = sum;
    __syncthreads();
    if (tid == 0) {
      float m = 0.f;
      for (int w = 0; w < kWarps; ++w) m += red_v[w];
      s_m = m;
    }
    __syncthreads();
  }

  // The next token, from the last accepted node's row.
  const int cur = s_cur;
  int next = 0;
  int odd = 0;
  if (!sample && is_inner(cur)) {
    next = best_of[cur];
  } else {
    const T* x = rows + (size_t)cur * p.V;
    const float* noise = sample ? p.noise + (size_t)r * p.V : nullptr;
    const float scale = p.inv_temp * kLog2e;
    float c = drafts ? s_c : 0.f;
    int ng = s_gone;
    while (true) {
      float v0 = -INFINITY;
      int i0 = p.V;
      if (!sample) {
        for_row<T, kWalkThreads>(x, 0, p.V, [&](int at, float v) {
          odd |= !(v < INFINITY);
          take_best(v0, i0, v, at);
        });
      } else if (c > 0.f) {
        const float* q = drafts + (size_t)cur * p.V;
        const float shift = lse[cur] * kLog2e;
        for_row<T, kWalkThreads>(x, 0, p.V, [&](int at, float v) {
          const float w = exp2f(v * scale - shift) - c * q[at];
          if (w > 0.f) take_best(v0, i0, w / noise[at], at);
        });
      } else {  // the whole row: in logarithms, so that no normaliser is needed
        for_row<T, kWalkThreads>(x, 0, p.V, [&](int at, float v) {
          odd |= !(v < INFINITY);
          bool out = v == -INFINITY;
          for (int e = 0; e < ng; ++e) out = out || gone[e] == at;
          if (!out) take_best(v0, i0, v * scale - log2f(noise[at]), at);
        });
      }
      warp_best(v0, i0);
      if (lane == 0) {
        red_v[warp] = v0;
        red_i[warp] = i0;
      }
      __syncthreads();
      if (warp == 0) {
        v0 = red_v[lane];
        i0 = red_i[lane];
        warp_best(v0, i0);
        if (lane == 0) red_i[0] = i0;
      }
      __syncthreads();
      next = red_i[0];
      if (next < p.V || (c == 0.f && ng == 0)) break;
      __syncthreads();
      c = 0.f;  // nothing left of the residual: the target itself
      ng = 0;
    }
    if (next >= p.V) odd = 1;
  }
  if (__syncthreads_or(odd)) {
    if (tid == 0) flag(p.dev_status, FLARE_DEV_BAD_LOGITS);
    return;
  }
  if (tid < p.N) {
    p.path[(size_t)r * p.N + tid] = tid < s_len ? line[tid] : -1;
    p.node_logp[(size_t)r * p.N + tid] = tid < n ? logp[tid] : 0.f;
  }
  if (tid == 0) {
    p.path_len[r] = s_len;
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
  if (p.N > 1) {  // a lone anchor has no row with children
    // rows along y: 65535 a launch
    TreeVerifyParams b = p;
    const int step = 65535 / p.N;  // requests per launch
    for (int r0 = 0; r0 < p.R; r0 += step) {
      const int nr = p.R - r0 < step ? p.R - r0 : step;
      const size_t e = (size_t)r0 * p.N;
      b.logits = static_cast<const T*>(p.logits) + e * p.V;
      b.parent = p.parent + e;
      b.node_len = p.node_len + r0;
      b.stats = p.stats + e * p.n_chunks;
      tree_rows_kernel<T>
          <<<dim3((unsigned)p.n_chunks, (unsigned)(nr * p.N)), kRowThreads, 0, stream>>>(b);
      note_launches(1);
      const cudaError_t err = cudaGetLastError();
      if (err != cudaSuccess) return err;
    }
  }
  tree_walk_kernel<T><<<(unsigned)p.R, kWalkThreads, 0, stream>>>(p);
  note_launches(1);
  return cudaGetLastError();
}
}  // namespace

cudaError_t launch_tree_verify(const TreeVerifyParams& p, bool bf16, cudaStream_t stream) {
  if (p.R == 0) return cudaSuccess;
  return bf16 ? launch_t<__nv_bfloat16>(p, stream) : launch_t<float>(p, stream);
}

}  // namespace flare
