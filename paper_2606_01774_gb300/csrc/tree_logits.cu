// Penalties for repeated tokens, biases and token masks on the logits of a tree's
// nodes.
//
// A CTA takes a chunk of the vocabulary and a share of a request's nodes.  What a
// token costs does not depend on the node, but for the few tokens that the tree
// itself holds: so the CTA counts the history's tokens of its chunk once, in
// shared memory, turns counts and biases into one summand per token, and streams
// its rows through.  The tree's own tokens are put right at the end, each by its
// count on every node's path.  Bound by bytes: logits in and out once.
#include "common.cuh"
#include "kernels.h"
#include "piece.cuh"
#include "tree.cuh"

namespace flare {

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kPrompt = 1u << 31;  // seen in the history ahead of the output; below: count

// Index of chunk token i: the eight tokens of a thread's piece, eight threads on, lie in
// banks of their own.
__device__ __forceinline__ int at(int i) { return i + (i >> 5); }

__device__ __forceinline__ float penalised(float x, bool seen, float rep, float rep_inv) {
  return seen ? (x > 0.f ? x * rep_inv : x * rep) : x;
}

__device__ __forceinline__ float minus_inf() { return __int_as_float(0xff800000); }

}  // namespace

template <typename T>
__global__ void __launch_bounds__(kThreads)
    tree_logits_kernel(const __grid_constant__ TreeLogitsParams p, int chunk, int chunks,
                       int row_parts) {
  constexpr int E = 16 / sizeof(T);  // elements of a piece
  extern __shared__ char smem[];
  float* add = reinterpret_cast<float*>(smem);                     // [at(chunk)]
  uint32_t* word = reinterpret_cast<uint32_t*>(smem);              // the same, while counting
  uint32_t* seen = reinterpret_cast<uint32_t*>(add + at(chunk));   // [chunk / 32] bits
  uint32_t* touched = seen + chunk / 32 + 1;  // seen, or with a summand (a word past the end: 0)
  __shared__ uint64_t path[kMaxNodes];
  __shared__ int tok[kMaxNodes];
  __shared__ uint32_t base[kMaxNodes];  // a node token's word
  __shared__ int tree_bad;

  const int tid = threadIdx.x, lane = tid & 31;
  const int team = blockIdx.x / chunks;
  const int r = team / row_parts, part = team - r * row_parts;
  const int c0 = (blockIdx.x - team * chunks) * chunk, c1 = min(c0 + chunk, p.V), len = c1 - c0;
  const int n = p.node_len ? p.node_len[r] : p.N;
  const int H = p.history ? p.history_len[r] : 0;
  const int out_from = p.history && p.output_start ? p.output_start[r] : 0;
  const int n_bias = p.bias_token ? p.bias_len[r] : 0;
  const float rep = p.repetition ? p.repetition[r] : 1.f;
  const float pres = p.presence ? p.presence[r] : 0.f;
  const float freq = p.frequency ? p.frequency[r] : 0.f;
  int bad = 0;
  if (n < 0 || n > p.N) bad |= FLARE_DEV_BAD_TREE;
  if (H < 0 || H > p.H || out_from < 0 || out_from > p.H || n_bias < 0 || n_bias > p.max_bias)
    bad |= FLARE_DEV_BAD_HISTORY;
  if (!(rep >= 0x1p-126f && rep < -minus_inf()) || !isfinite(pres) || !isfinite(freq))
    bad |= FLARE_DEV_BAD_PENALTY;
  if (bad) {
    if (tid == 0) flag(p.dev_status, bad);
    return;
  }
  const bool tree = p.token != nullptr;

  for (int i = tid; i < at(chunk); i += kThreads) word[i] = 0;
  if (tid < 32) {  // the tree's paths and tokens
    bool ok = true;
    if (tree) {
      int p0, p1;
      uint64_t a0, a1;
      ok = warp_load_tree(p.parent + (size_t)r * p.N, n, p0, p1);
      if (ok) {
        warp_paths(n, p0, p1, a0, a1);
        path[lane] = a0;
        path[lane + 32] = a1;
      }
      for (int i = lane; i < n; i += 32) {
        const int x = p.token[(size_t)r * p.N + i];
        tok[i] = x;
        ok = ok && x >= 0 && x < p.V;
      }
    }
    ok = __all_sync(0xffffffffu, ok);
    if (lane == 0) tree_bad = !ok;
  }
  __syncthreads();
  if (tree_bad) {
    if (tid == 0) flag(p.dev_status, FLARE_DEV_BAD_TREE);
    return;
  }
  const int32_t* hist = p.history ? p.history + (size_t)r * p.H : nullptr;
  int wrong = 0;
  for (int i = tid; i < H; i += kThreads) {
    const int x = hist[i];
    wrong |= x < 0 || x >= p.V;
    if (x >= c0 && x < c1) {
      if (i >= out_from) atomicAdd(&word[at(x - c0)], 1u);
      else atomicOr(&word[at(x - c0)], kPrompt);
    }
  }
  const int32_t* bias_token = p.bias_token ? p.bias_token + (size_t)r * p.max_bias : nullptr;
  const float* bias_value = p.bias_token ? p.bias_value + (size_t)r * p.max_bias : nullptr;
  for (int i = tid; i < n_bias; i += kThreads)
    wrong |= bias_token[i] < 0 || bias_token[i] >= p.V;
  if (__syncthreads_or(wrong)) {
    if (tid == 0) flag(p.dev_status, FLARE_DEV_BAD_HISTORY);
    return;
  }
  // the tree's tokens pass the rows below as they are: no count, no summand but the bias
  const bool held = tree && tid < n && tok[tid] >= c0 && tok[tid] < c1;
  if (held) base[tid] = word[at(tok[tid] - c0)];
  __syncthreads();
  if (held) word[at(tok[tid] - c0)] = 0;
  __syncthreads();
  for (int i0 = 0; i0 < chunk; i0 += kThreads) {  // counts to summands, in place
    const int i = i0 + tid;
    const uint32_t w = word[at(i)];
    const uint32_t c = w & ~kPrompt;
    const float s = c ? -freq * (float)c - pres : 0.f;
    add[at(i)] = s;
    const uint32_t any = __ballot_sync(0xffffffffu, w != 0);
    if (lane == 0) seen[i >> 5] = touched[i >> 5] = any;
  }
  if (tid == 0) touched[chunk / 32] = 0;
  __syncthreads();
  if (tid < 32) {  // biases in the list's order, a token's repetitions one after another
    for (int i0 = 0; i0 < n_bias; i0 += 32) {
      const int x = i0 + lane < n_bias ? bias_token[i0 + lane] : -1;
      const bool mine = x >= c0 && x < c1;
      const float b = mine ? bias_value[i0 + lane] : 0.f;
      const uint32_t same = __match_any_sync(0xffffffffu, mine ? x : -1 - lane);
      float sum = mine ? add[at(x - c0)] : 0.f;
      if (__all_sync(0xffffffffu, same == 1u << lane)) {
        sum += b;
      } else {
        for (int src = 0; src < 32; ++src) {
          const float other = __shfl_sync(0xffffffffu, b, src);
          if (same >> src & 1) sum += other;
        }
      }
      if (mine && lane == __ffs(same) - 1) {
        add[at(x - c0)] = sum;
        atomicOr(&touched[(x - c0) >> 5], 1u << ((x - c0) & 31));
      }
      __syncwarp();
    }
  }
  __syncthreads();
  if (held) atomicAnd(&touched[(tok[tid] - c0) >> 5], ~(1u << ((tok[tid] - c0) & 31)));
  __syncthreads();

  const float rep_inv = 1.f / rep;
  const float none = minus_inf();
  const int mask_words = (p.V + 31) / 32;
  const bool in_place = p.logits == p.out;
  const int row_first = (int)((long long)n * part / row_parts);
  const int row_last = (int)((long long)n * (part + 1) / row_parts);
  for (int i = row_first; i < row_last; ++i) {
    const size_t row = (size_t)r * p.N + i;
    const T* src = static_cast<const T*>(p.logits) + row * p.V + c0;
    T* dst = static_cast<T*>(p.out) + row * p.V + c0;
    const uint32_t* mask = p.mask ? p.mask + row * mask_words : nullptr;
    const bool together = ((uintptr_t)src & 15) == ((uintptr_t)dst & 15);
    // elements ahead of the first whole piece: all of them where the rows' 16-byte grids differ
    const int ahead = (int)((16 - ((uintptr_t)src & 15)) & 15) / (int)sizeof(T);
    const int head = together ? min(len, ahead) : len;
    const int pieces = (len - head) / E;
    for (int j = tid; j < pieces; j += kThreads) {
      const int e = head + j * E;
      uint32_t m = (1u << E) - 1;  // allowed
      if (mask) {
        const int b = c0 + e, w = b >> 5;
        const uint32_t next = w + 1 < mask_words ? mask[w + 1] : 0;
        m &= __funnelshift_r(mask[w], next, b & 31);
      }
      const uint32_t t =
          __funnelshift_r(touched[e >> 5], touched[(e >> 5) + 1], e & 31) & ((1u << E) - 1);
      if (in_place && m == (1u << E) - 1 && !t) continue;
      uint4 raw;
      if (m) raw = *reinterpret_cast<const uint4*>(src + e);
      if (t || m != (1u << E) - 1) {
        float x[E];
        Piece<T>::load(raw, x);
        const uint32_t sn = __funnelshift_r(seen[e >> 5], seen[(e >> 5) + 1], e & 31);
#pragma unroll
        for (int k = 0; k < E; ++k) {
          if (t >> k & 1) x[k] = penalised(x[k], sn >> k & 1, rep, rep_inv) + add[at(e + k)];
          if (!(m >> k & 1)) x[k] = none;
        }
        raw = Piece<T>::store(x);
      }
      *reinterpret_cast<uint4*>(dst + e) = raw;
    }
    // the ends that are no whole piece
    const int rest = len - pieces * E;
    for (int j = tid; j < rest; j += kThreads) {
      const int e = j < head ? j : j + pieces * E;
      const bool ok = !mask || mask[(c0 + e) >> 5] >> ((c0 + e) & 31) & 1;
      const bool change = touched[e >> 5] >> (e & 31) & 1;
      if (in_place && ok && !change) continue;
      float x = none;
      if (ok) {
        x = to_f32(src[e]);
        if (change)
          x = penalised(x, seen[e >> 5] >> (e & 31) & 1, rep, rep_inv) + add[at(e)];
      }
      dst[e] = from_f32<T>(x);
    }
  }
  if (!tree) return;
  __syncthreads();

  // the tree's tokens: each row by its own path's count
  const int rows = row_last - row_first;
  for (int j = tid; j < rows * n; j += kThreads) {
    const int i = row_first + j / n, m = j % n, x = tok[m];
    if (x < c0 || x >= c1) continue;
    uint64_t same = 0;
    for (int k = 0; k < n; ++k) same |= (uint64_t)(tok[k] == x) << k;
    if (m != __ffsll(same) - 1) continue;  // once
    const size_t row = (size_t)r * p.N + i;
    if (p.mask && !(p.mask[row * mask_words + (x >> 5)] >> (x & 31) & 1)) continue;
    const int mine = __popcll(same & path[i]);
    const uint32_t c = (base[m] & ~kPrompt) + mine;
    float y = to_f32(static_cast<const T*>(p.logits)[row * p.V + x]);
    y = penalised(y, base[m] != 0 || mine, rep, rep_inv);
    if (c) y -= freq * (float)c + pres;
    static_cast<T*>(p.out)[row * p.V + x] = from_f32<T>(y + add[at(x - c0)]);
  }
}

cudaError_t launch_tree_logits(const TreeLogitsParams& p, bool bf16, int num_sms,
                               cudaStream_t stream) {
  if (p.R == 0) return cudaSuccess;
  // the largest chunk that still gives every SM several CTAs
  int chunk = 4096;
  while (chunk > 512 && (int64_t)p.R * ((p.V + chunk - 1) / chunk) < 3 * num_sms) chunk /= 2;
  const int chunks = (p.V + chunk - 1) / chunk;
  int parts = 1;
  while (parts * 2 <= p.N && (int64_t)p.R * chunks * parts < 2 * num_sms) parts *= 2;
  if ((int64_t)p.R * parts * chunks > INT32_MAX) return cudaErrorInvalidConfiguration;
  const int smem = (chunk + chunk / 32 + 2 * (chunk / 32 + 1)) * 4;
  const unsigned grid = (unsigned)p.R * parts * chunks;
  if (bf16)
    tree_logits_kernel<__nv_bfloat16><<<grid, kThreads, smem, stream>>>(p, chunk, chunks, parts);
  else
    tree_logits_kernel<float><<<grid, kThreads, smem, stream>>>(p, chunk, chunks, parts);
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace flare
