// Penalties for repeated tokens, biases and token masks on the logits of a tree's nodes.
//
//   y = l (l > 0 ? up : down) + add      up, down: 1 / repetition and repetition where the token was
//                                        seen, else 1; add: -frequency c - presence [c > 0] + bias
//
// A CTA takes a chunk of the vocabulary and a share of a request's nodes.  What a token gets does
// not depend on the node, but for the few tokens that the tree itself holds: so the CTA counts
// the history's tokens of its chunk once, in shared memory, and streams its rows through.  A lane
// has the same tokens in every row and finds out once what they get.  Tokens that are neither
// seen nor biased (a bit each) cost nothing but their copy, in place not even that.  The tree's
// own tokens come last, each by its count on every node's path.
//
// Bound by bytes once there are many rows, logits in and out (64 requests x 64 nodes over 32000
// bf16 tokens: 99 us, 5.3 TB/s, under a mask 102); with few, by the steps before them: lengths,
// tree, history and biases are round trips to memory one after another, some 3 us, and a history of
// 8192 tokens is counted once per chunk, 3 us of 34 for 64 x 16 nodes under a mask (4.1 TB/s), 9 of
// 24 for 64 x 1 over 128000.  One wave of three CTAs an SM keeps that to once; with two these take 40
// and 28 us.  Some masked forms and those for one or two fp32 rows pass what 80 registers a thread
// do not hold through local memory (12 to 308 bytes); with registers for two CTAs an SM, where
// nothing does, the two calls take 39 and 26 us.
#pragma once

#include "common.cuh"
#include "kernels.h"
#include "piece.cuh"
#include "tree.cuh"

namespace flare {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kCtas = 3;                 // of an SM
template <typename T>
constexpr int kRowsOf = sizeof(T) == 2 ? 3 : 2;  // more take registers that a third CTA needs
constexpr int kScan = 8;                 // pieces of the history in flight per thread, four tokens each
constexpr uint32_t kPrompt = 1u << 31;   // seen in the history ahead of the output; below: count
constexpr int kSmemMost = 220 << 10;     // of a CTA, besides the static part
constexpr int kAhead = 32 << 10;         // bytes of the rows that a CTA asks into L2
constexpr int kNarrow = 32767;           // the longest history whose counts have 16 bits each

// Index of chunk token i: the eight tokens of a thread's piece, eight threads on, lie in
// banks of their own.
__host__ __device__ __forceinline__ int at(int i) { return i + (i >> 5); }

__device__ __forceinline__ float minus_inf() { return __int_as_float(0xff800000); }

// Bits i .. i + 31 of a bit array (which ends with a word to spare).
__device__ __forceinline__ uint32_t bits_at(const uint32_t* bits, int i) {
  return __funnelshift_r(bits[i >> 5], bits[(i >> 5) + 1], i & 31);
}

// A piece's words where its tokens are allowed, by their bits: ones, else zeros.
template <typename T>
__device__ __forceinline__ uint4 keep_words(uint32_t allowed) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 2)
      w[i] = (allowed >> (2 * i) & 1 ? 0xffffu : 0u) | (allowed >> (2 * i) & 2 ? 0xffff0000u : 0u);
    else
      w[i] = allowed >> i & 1 ? ~0u : 0u;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// `raw` with -inf where `keep` is zeros.
template <typename T>
__device__ __forceinline__ uint4 ruled_out(const uint4& raw, const uint4& keep) {
  const uint32_t none = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
  return make_uint4((raw.x & keep.x) | (none & ~keep.x), (raw.y & keep.y) | (none & ~keep.y),
                    (raw.z & keep.z) | (none & ~keep.z), (raw.w & keep.w) | (none & ~keep.w));
}

// How often the history holds each token of a chunk: in the output, with kPrompt where the prompt has
// it too.  Two tokens to a word where the history is short.
struct Counts {
  uint32_t* word;
  bool narrow;

  __device__ __forceinline__ uint32_t full(int e) const { return word[at(e)]; }
  __device__ __forceinline__ uint32_t half(int e) const {
    const uint32_t w = word[at(e >> 1)] >> (e & 1) * 16;
    return (w & 0x7fffu) | (w & 0x8000u) << 16;
  }
  __device__ __forceinline__ uint32_t operator[](int e) const { return narrow ? half(e) : full(e); }
  __device__ __forceinline__ void add(int e, bool output) const {
    uint32_t* w = &word[at(narrow ? e >> 1 : e)];
    const int shift = narrow ? (e & 1) * 16 : 0;
    if (output) atomicAdd(w, 1u << shift);
    else atomicOr(w, narrow ? 0x8000u << shift : kPrompt);
  }
};

// What a piece's tokens get: y = x (x > 0 ? up : down) + add, which leaves what is neither seen
// nor has a summand as it is (x + -0 is x, for both zeros).
template <int E>
struct Change {
  float up[E], down[E], add[E];
};

// A request's penalties, and its history's counts and biases over a chunk of the vocabulary.
struct Tables {
  float rep, rep_inv, pres, freq;
  Counts counts;
  const uint32_t* biased;  // [chunk / 32] bits: tokens with a bias
  const uint32_t* before;  // [chunk / 32] how many bits are set in the words before
  const float* bias;       // of the tokens with one, in order

  __device__ __forceinline__ float bias_of(int e) const {
    const uint32_t w = biased[e >> 5], bit = 1u << (e & 31);
    return w & bit ? bias[before[e >> 5] + __popc(w & (bit - 1))] : -0.f;
  }

  // What a count does to its token.
  __device__ __forceinline__ void one(uint32_t w, float& up, float& down, float& add) const {
    const uint32_t c = w & ~kPrompt;
    up = w ? rep_inv : 1.f;
    down = w ? rep : 1.f;
    add = c ? -freq * (float)c - pres : -0.f;
  }
  // Of a piece whose element k is token e + k / S * 32 S + k % S (GRID: e a multiple of S).  All
  // counts are asked for before the first is used: a warp whose piece is touched in every row
  // holds up its CTA.
  template <int E, int S, bool GRID>
  __device__ __forceinline__ void piece(int e, uint32_t touched, Change<E>& ch) const {
    uint32_t w[E], some = 0;
    if (counts.narrow) {
#pragma unroll
      for (int k = 0; k < E; ++k)
        w[k] = touched >> k & 1 ? counts.half(e + k / S * 32 * S + k % S) : 0;
    } else {
#pragma unroll
      for (int k = 0; k < E; ++k)
        w[k] = touched >> k & 1 ? counts.full(e + k / S * 32 * S + k % S) : 0;
    }
#pragma unroll
    for (int k = 0; k < E; k += S) {
      const int x = e + k * 32;
      const uint32_t bits = GRID ? biased[x >> 5] >> (x & 31) : bits_at(biased, x);
      some |= (bits & ((1u << S) - 1)) << k;
    }
#pragma unroll
    for (int k = 0; k < E; ++k) one(w[k], ch.up[k], ch.down[k], ch.add[k]);
    if (some & touched) {
#pragma unroll
      for (int k = 0; k < E; ++k)
        if (some & touched & 1u << k) ch.add[k] += bias_of(e + k / S * 32 * S + k % S);
    }
  }
};

template <typename T, int E>
__device__ __forceinline__ uint4 changed(const uint4& raw, const Change<E>& ch) {
  float x[E];
  Piece<T>::load(raw, x);
#pragma unroll
  for (int k = 0; k < E; ++k) x[k] = fmaf(x[k], x[k] > 0.f ? ch.up[k] : ch.down[k], ch.add[k]);
  return Piece<T>::store(x);
}

// W consecutive bytes of a row, a part of a piece.
template <int W>
struct Part;
template <>
struct Part<16> {
  using Type = uint4;
};
template <>
struct Part<8> {
  using Type = uint2;
};
template <>
struct Part<4> {
  using Type = uint32_t;
};

template <int W>
__device__ __forceinline__ void get_part(uint4& raw, int k, const void* from) {
  uint32_t* w = reinterpret_cast<uint32_t*>(&raw);
  const auto v = *static_cast<const typename Part<W>::Type*>(from);
  if constexpr (W == 16) raw = v;
  if constexpr (W == 8) w[2 * k] = v.x, w[2 * k + 1] = v.y;
  if constexpr (W == 4) w[k] = v;
}

template <int W>
__device__ __forceinline__ void put_part(const uint4& raw, int k, void* to) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&raw);
  if constexpr (W == 16) *static_cast<uint4*>(to) = raw;
  if constexpr (W == 8) *static_cast<uint2*>(to) = make_uint2(w[2 * k], w[2 * k + 1]);
  if constexpr (W == 4) *static_cast<uint32_t*>(to) = w[k];
}

// The pieces of a warp's lanes in ROWS rows: taken in, then changed, ruled out and put back.
// `live`: the piece's elements inside the chunk, a whole number of parts.
template <typename T, int W, int ROWS, bool MASK, bool IN_PLACE>
struct Batch {
  static constexpr int E = Piece<T>::N, S = W / (int)sizeof(T), K = E / S;
  uint4 raw[ROWS];
  uint32_t word[ROWS][MASK ? K : 1];  // the mask's bytes, untouched while they are on their way

  // Which of row u's tokens are allowed, `bit` the first one's place in its byte.
  __device__ __forceinline__ uint32_t allowed(int u, int bit, uint32_t live) const {
    if (!MASK) return live;
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) bits |= (word[u][k] >> bit & ((1u << S) - 1)) << (k * S);
    return bits;
  }
  // src: the lane's first element, bits: the mask's byte with it, both of the first row.
  __device__ __forceinline__ void load(const T* src, size_t V, const uint8_t* bits, int bit,
                                       size_t mask_bytes, uint32_t live, bool kept) {
    if (MASK) {
#pragma unroll
      for (int u = 0; u < ROWS; ++u)
#pragma unroll
        for (int k = 0; k < K; ++k)
          word[u][k] = live >> (k * S) & 1 ? bits[u * mask_bytes + k * 4 * S] : 0;
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      // what stays as it is, stays
      if (IN_PLACE && kept && (!MASK || allowed(u, bit, live) == live)) continue;
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (live >> (k * S) & 1) get_part<W>(raw[u], k, src + u * V + k * 32 * S);
    }
  }
  __device__ __forceinline__ void store(T* dst, size_t V, int bit, const uint4* keep_of,
                                        uint32_t touched, const Change<E>& ch, uint32_t live,
                                        bool kept) {
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      const uint32_t ok = allowed(u, bit, live);
      if (IN_PLACE && kept && ok == live) continue;
      if (touched & ok) raw[u] = changed<T>(raw[u], ch);
      if (MASK) raw[u] = ruled_out<T>(raw[u], keep_of[ok]);
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (live >> (k * S) & 1) put_part<W>(raw[u], k, dst + u * V + k * 32 * S);
    }
  }
};

}  // namespace

// W: bytes on whose boundaries all rows start, up to 16.  A lane's piece is 16 bytes in parts of W, a
// warp's parts next to each other: the same tokens in every row, whatever V is.  (fp32 parts of 4
// against W = 0, 9 trees of 13 over 50257 tokens: 11 us, 12.)  W = 0, for bf16 rows on 2 or 4
// bytes: pieces start at each row's own 16-byte boundaries and look up their tokens in each (parts
// of 2, 4 trees of 26 over 81625: 34 us, 25 at the time and now 14).  FEW: rows too few to keep a
// batch under way, so several blocks of a row are (64 x 1 over 128000: 24 us, 29 without).
template <typename T, int W, bool MASK, bool IN_PLACE, bool FEW>
__global__ void __launch_bounds__(kThreads, kCtas)
    tree_logits_kernel(const __grid_constant__ TreeLogitsParams p, int chunk, int chunks,
                       int row_parts, bool narrow) {
  constexpr int E = Piece<T>::N;               // elements of a piece
  // In flight per thread, twice.  W = 0 has to remember more with each (three: 44 us, two: 36, for 16
  // trees of 36 nodes over 52711 tokens under a mask).
  constexpr int kRows = W ? kRowsOf<T> : 2;
  constexpr uint32_t kFull = (1u << E) - 1;
  constexpr int S = W ? W / (int)sizeof(T) : E;  // of a part
  extern __shared__ __align__(16) char smem[];
  const Counts counts{reinterpret_cast<uint32_t*>(smem), narrow};
  const int count_words = at(narrow ? chunk / 2 : chunk);
  const int bit_words = chunk / 32 + 1;                // a word to spare
  uint32_t* touched = counts.word + count_words;  // bits: seen in the history or with a bias
  uint32_t* held = touched + bit_words;  // the tree's own tokens, which come last
  uint32_t* biased = held + bit_words;
  uint32_t* before = biased + bit_words;  // see Tables
  float* bias = reinterpret_cast<float*>(before + bit_words);  // [min(chunk, max_bias)]
  __shared__ uint64_t path[kMaxNodes];
  __shared__ int tok[kMaxNodes];
  __shared__ uint4 keep_of[1 << E];  // keep_words
  __shared__ int tree_bad, owns;
  __shared__ uint64_t own_nodes[kMaxNodes];  // of the tree's own tokens in the chunk: who has them
  __shared__ int own_token[kMaxNodes];       // and which they are, `owns` of them

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
  const int row_first = (int)((long long)n * part / row_parts);
  const int row_last = (int)((long long)n * (part + 1) / row_parts);
  const T* logits = static_cast<const T*>(p.logits) + (size_t)r * p.N * p.V + c0;
  T* out = static_cast<T*>(p.out) + (size_t)r * p.N * p.V + c0;

  // The history's first pieces are asked for ahead of the rows, which keep the memory busy.
  const int32_t* hist = p.history ? p.history + (size_t)r * p.H : nullptr;
  const bool quads = ((uintptr_t)hist & 15) == 0;
  int4 text[kScan];
  const auto take = [&](int i0) {  // a thread's tokens i0 .. i0 + 3, and so on a round further
#pragma unroll
    for (int j = 0; j < kScan; ++j) {
      const int i = i0 + j * 4 * kThreads;
      if (quads && i + 4 <= H) {
        text[j] = *reinterpret_cast<const int4*>(hist + i);
      } else {
        text[j].x = i < H ? hist[i] : 0;
        text[j].y = i + 1 < H ? hist[i + 1] : 0;
        text[j].z = i + 2 < H ? hist[i + 2] : 0;
        text[j].w = i + 3 < H ? hist[i + 3] : 0;
      }
    }
  };
  take(4 * tid);
  // and so are the first biases, by the warp that takes them
  const int32_t* bias_token = p.bias_token + (size_t)r * p.max_bias;
  const float* bias_value = p.bias_value + (size_t)r * p.max_bias;
  int pick[2] = {};
  float pick_value[2] = {};
  if (p.bias_token && tid >= kThreads - 32) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (lane + 32 * k < p.max_bias)
        pick[k] = bias_token[lane + 32 * k], pick_value[k] = bias_value[lane + 32 * k];
  }
  for (int i = tid; i < (count_words + 4 * bit_words + 3) / 4; i += kThreads)  // room for all of it
    reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
  if (tid < 1 << E) keep_of[tid] = keep_words<T>(tid);

  if (tid < 32) {  // the tree's paths and tokens
    bool ok = true;
    if (tree) {
      const int32_t* token = p.token + (size_t)r * p.N;
      const int x0 = lane < n ? token[lane] : 0, x1 = lane + 32 < n ? token[lane + 32] : 0;
      int p0, p1;
      uint64_t a0, a1;
      ok = warp_load_tree(p.parent + (size_t)r * p.N, n, p0, p1);
      if (ok) {
        warp_paths(n, p0, p1, a0, a1);
        path[lane] = a0;
        path[lane + 32] = a1;
      }
      tok[lane] = x0;
      tok[lane + 32] = x1;
      ok = ok && (uint32_t)x0 < (uint32_t)p.V && (uint32_t)x1 < (uint32_t)p.V;
    }
    ok = __all_sync(0xffffffffu, ok);
    if (lane == 0) tree_bad = !ok, owns = 0;
  }
  __syncthreads();
  if (tree_bad) {
    if (tid == 0) flag(p.dev_status, FLARE_DEV_BAD_TREE);
    return;
  }
  if (!IN_PLACE || MASK) {
    // the first rows, on their way to L2 while the history is counted (ahead of the loads above they
    // would only hold those up)
    const int first_rows = min(row_last - row_first, kAhead / (len * (int)sizeof(T)));
    for (int i = row_first + tid; i < row_first + first_rows; i += kThreads) {
      const uintptr_t row = (uintptr_t)(logits + (size_t)i * p.V), from = row & ~(uintptr_t)15;
      const uint32_t bytes = (uint32_t)(row + len * sizeof(T) - from) & ~15u;
      if (bytes)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"(bytes)
                     : "memory");
    }
  }
  int wrong = 0;
  const auto count = [&](int i, int x) {
    wrong |= (uint32_t)x >= (uint32_t)p.V;
    const int e = x - c0;
    if ((uint32_t)e >= (uint32_t)len) return;
    counts.add(e, i >= out_from);
    atomicOr(&touched[e >> 5], 1u << (e & 31));
  };
  for (int i0 = 4 * tid; i0 < H; i0 += 4 * kThreads * kScan) {
    if (i0 >= 4 * kThreads * kScan) take(i0);
#pragma unroll
    for (int j = 0; j < kScan; ++j) {
      const int i = i0 + j * 4 * kThreads;
      if (i >= H) break;
      count(i, text[j].x);
      if (i + 1 < H) count(i + 1, text[j].y);
      if (i + 2 < H) count(i + 2, text[j].z);
      if (i + 3 < H) count(i + 3, text[j].w);
    }
  }
  if (tree && tid < n && tok[tid] >= c0 && tok[tid] < c1) {
    const int x = tok[tid], e = x - c0;
    uint64_t same = 0;
#pragma unroll 8
    for (int k = 0; k < n; ++k) same |= (uint64_t)(tok[k] == x) << k;
    if (tid == __ffsll(same) - 1) {  // once
      const int i = atomicAdd(&owns, 1);
      own_nodes[i] = same;
      own_token[i] = e;
      atomicOr(&held[e >> 5], 1u << (e & 31));
    }
  }
  if (tid >= kThreads - 32) {
    // biases by one warp: which tokens have one, and then the list in its order, a token's repetitions
    // one after another
    bool any = false;
    for (int i = lane; i < n_bias; i += 32) {
      const int x = i < 32 ? pick[0] : i < 64 ? pick[1] : bias_token[i], e = x - c0;
      wrong |= (uint32_t)x >= (uint32_t)p.V;
      if ((uint32_t)e >= (uint32_t)len) continue;
      any = true;
      atomicOr(&biased[e >> 5], 1u << (e & 31));
    }
    __syncwarp();  // every lane's bits, before others read them: a vote orders no memory
    if (__any_sync(0xffffffffu, any)) {
      uint32_t total = 0;
      for (int i0 = 0; i0 < bit_words; i0 += 32) {
        const uint32_t own = i0 + lane < bit_words ? __popc(biased[i0 + lane]) : 0;
        uint32_t sum = own;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
          const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
          if (lane >= o) sum += up;
        }
        if (i0 + lane < bit_words) before[i0 + lane] = total + sum - own;
        total += __shfl_sync(0xffffffffu, sum, 31);
      }
      for (uint32_t i = lane; i < total; i += 32) bias[i] = 0.f;
      __syncwarp();
      for (int i0 = 0; i0 < n_bias; i0 += 32) {
        const int i = i0 + lane;
        const int e = i < n_bias ? (i < 32 ? pick[0] : i < 64 ? pick[1] : bias_token[i]) - c0 : -1;
        const bool mine = (uint32_t)e < (uint32_t)len;
        const float b = !mine ? 0.f : i < 32 ? pick_value[0] : i < 64 ? pick_value[1] : bias_value[i];
        const uint32_t w = mine ? biased[e >> 5] : 0, bit = 1u << (e & 31);
        float* const sum = bias + (mine ? before[e >> 5] + __popc(w & (bit - 1)) : 0);
        float value = mine ? *sum : 0.f;
        const uint32_t same = __match_any_sync(0xffffffffu, mine ? e : -1 - lane);
        if (__all_sync(0xffffffffu, same == 1u << lane)) {
          value += b;
        } else {
          for (int src = 0; src < 32; ++src) {
            const float other = __shfl_sync(0xffffffffu, b, src);
            if (same >> src & 1) value += other;
          }
        }
        if (mine && lane == __ffs(same) - 1) *sum = value;
        __syncwarp();
      }
    }
  }
  if (__syncthreads_or(wrong)) {
    if (tid == 0) flag(p.dev_status, FLARE_DEV_BAD_HISTORY);
    return;
  }
  for (int i = tid; i < bit_words; i += kThreads) touched[i] = (touched[i] | biased[i]) & ~held[i];
  __syncthreads();

  const Tables tables{rep, 1.f / rep, pres, freq, counts, biased, before, bias};
  const int mask_words = (p.V + 31) / 32;
  const uint32_t* mask = p.mask ? p.mask + (size_t)r * p.N * mask_words : nullptr;
  // Warps side by side take the chunk's blocks of 32 pieces, kRows rows at a time: all warps while
  // there are blocks for all.  For the rest as many warps side by side as make the fewest steps,
  // the others taking other rows.
  const auto each_block = [&](const auto& rows_of) {
    const int blocks = (len + 32 * E - 1) / (32 * E), full = blocks / kWarps * kWarps;
    int from = 0, side = kWarps;
    while (from < blocks) {
      const int to = from < full ? full : blocks;
      if (from == full) {
        int fewest = INT32_MAX;
#pragma unroll
        for (int s = kWarps; s > 0; s /= 2) {
          const int step = kWarps / s * kRows;
          const int steps = ((to - from + s - 1) / s) * ((row_last - row_first + step - 1) / step);
          if (steps < fewest) side = s, fewest = steps;
        }
      }
      const int group = tid / 32 / side;
      for (int block = from + tid / 32 % side; block < to; block += side)
        rows_of(block * 32 * E, row_first + group * kRows, kWarps / side * kRows);
      from = to;
    }
  };
  const size_t V = p.V, mask_bytes = (size_t)mask_words * 4;
  if constexpr (W == 0) {
    const bool together = ((uintptr_t)logits & 15) == ((uintptr_t)out & 15);
    const auto words_at = [&](int row, int e, uint32_t& first, uint32_t& next) {
      if (!MASK) return;
      const uint32_t* w = mask + (size_t)row * mask_words + ((c0 + e) >> 5);
      first = w[0];
      next = w[((c0 + e) >> 5) + 1 < mask_words];  // past the last: the last again, not used
    };
    const auto allowed_of = [&](int e, uint32_t first, uint32_t next) -> uint32_t {
      return MASK ? __funnelshift_r(first, next, (c0 + e) & 31) & kFull : kFull;
    };
    // every row its own grid: the pieces start at its first 16-byte boundary
    const auto ahead = [&](int i) {
      const uintptr_t first = (uintptr_t)(logits + (size_t)i * p.V) & 15;
      return min(len, (int)((16 - first) & 15) / (int)sizeof(T));
    };
    // A warp takes an equal share of all rows' blocks one after another, kRows of them at a time, so
    // that blocks with many tokens to change are spread over the warps.
    const int blocks = (len + 32 * E - 1) / (32 * E), items = (row_last - row_first) * blocks;
    const int share = (items + kWarps - 1) / kWarps;
    int item = tid / 32 * share, row = row_first + item / blocks, block = item % blocks;
    const int last = together ? min(item + share, items) : 0;
    struct {
      uint4 raw[kRows];
      uint32_t word[2][kRows], touched[kRows];  // of the mask, as they came
      int row[kRows], e[kRows];
    } one, two;
    const auto load = [&](auto& batch) {  // the next items
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int i = row, e = item < last ? ahead(i) + (block * 32 + lane) * E : len;
        if (++block == blocks) block = 0, ++row;
        ++item;
        batch.row[u] = i;
        batch.e[u] = e;
        if (e + E > len) continue;
        batch.touched[u] = bits_at(touched, e) & kFull;
        uint32_t &w0 = batch.word[0][u], &w1 = batch.word[1][u];
        words_at(i, e, w0, w1);
        if (!(IN_PLACE && !batch.touched[u] && allowed_of(e, w0, w1) == kFull))
          batch.raw[u] = *reinterpret_cast<const uint4*>(logits + i * V + e);
      }
    };
    const auto store = [&](auto& batch) {
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int i = batch.row[u], e = batch.e[u];
        if (e + E > len) continue;
        const uint32_t m = allowed_of(e, batch.word[0][u], batch.word[1][u]), t = batch.touched[u];
        if (IN_PLACE && m == kFull && !t) continue;
        if (t & m) {
          Change<E> ch;
          tables.piece<E, E, false>(e, t & m, ch);
          batch.raw[u] = changed<T>(batch.raw[u], ch);
        }
        if (MASK) batch.raw[u] = ruled_out<T>(batch.raw[u], keep_of[m]);
        *reinterpret_cast<uint4*>(out + i * V + e) = batch.raw[u];
      }
    };
    for (load(one); item - kRows < last; ) {
      load(two);
      store(one);
      if (item - kRows >= last) break;
      load(one);
      store(two);
    }
    const auto element = [&](int i, int e) {
      const T x_in = logits[(size_t)i * p.V + e];
      uint32_t w0, w1;
      words_at(i, e, w0, w1);
      const bool ok = allowed_of(e, w0, w1) & 1, changes = touched[e >> 5] >> (e & 31) & 1;
      if (IN_PLACE && ok && !changes) return;
      float x = ok ? to_f32(x_in) : minus_inf();
      if (ok && changes) {
        float up, down, add;
        tables.one(counts[e], up, down, add);
        add += tables.bias_of(e);
        x = fmaf(x, x > 0.f ? up : down, add);
      }
      out[(size_t)i * p.V + e] = from_f32<T>(x);
    };
    if (together) {  // the ends that are no whole piece, fewer than E on each side
      for (int k = tid; k < (row_last - row_first) * 2 * E; k += kThreads) {
        const int i = row_first + k / (2 * E), j = k % (2 * E);
        const int head = ahead(i), pieces = (len - head) / E, rest = len - pieces * E;
        if (j < rest) element(i, j < head ? j : j + pieces * E);
      }
    } else {
      for (int i = row_first; i < row_last; ++i)
        for (int e = tid; e < len; e += kThreads) element(i, e);
    }
  } else {
    // of a lane's piece: the elements in the chunk (V is a whole number of parts), and those to change
    const auto bits_of = [&](int e, uint32_t& live, uint32_t& t) {
      live = t = 0;
#pragma unroll
      for (int k = 0; k < E; k += S) {
        const int x = e + k * 32;
        if (x >= len) continue;
        live |= ((1u << S) - 1) << k;
        t |= (touched[x >> 5] >> (x & 31) & ((1u << S) - 1)) << k;
      }
    };
    if constexpr (FEW) {  // several blocks of a row under way together
      constexpr int kBlocks = 4;
      const int stride = kThreads * E;
      for (int i = row_first; i < row_last; ++i) {
        for (int block = tid / 32 * 32 * E; block < len; block += kBlocks * stride) {
          Batch<T, W, 1, MASK, IN_PLACE> batch[kBlocks];
          uint32_t live[kBlocks], t[kBlocks];
          const T* src = logits + i * V + block + lane * S;
          T* dst = out + i * V + block + lane * S;
          const uint8_t* bits = reinterpret_cast<const uint8_t*>(mask) + i * mask_bytes +
                                (c0 + block + lane * S) / 8;
#pragma unroll
          for (int u = 0; u < kBlocks; ++u) {
            bits_of(block + u * stride + lane * S, live[u], t[u]);
            batch[u].load(src + u * stride, V, bits + u * stride / 8, lane * S & 7, mask_bytes,
                          live[u], !t[u]);
          }
#pragma unroll
          for (int u = 0; u < kBlocks; ++u) {
            Change<E> ch;
            if (t[u]) tables.piece<E, S, true>(block + u * stride + lane * S, t[u], ch);
            batch[u].store(dst + u * stride, V, lane * S & 7, keep_of, t[u], ch, live[u], !t[u]);
          }
        }
      }
    } else {
      each_block([&](int block, int i, int step) {
        const int e = block + lane * S;
        uint32_t live, t;
        bits_of(e, live, t);
        if (S == E) {
          if (!live) return;
          live = kFull;
        }
        Change<E> ch;
        if (t) tables.piece<E, S, true>(e, t, ch);
        const bool kept = !t;
        const uint8_t* bits = reinterpret_cast<const uint8_t*>(mask) + (c0 + e) / 8;
        const auto load = [&](auto& batch, int i) {
          batch.load(logits + i * V + e, V, bits + i * mask_bytes, e & 7, mask_bytes, live, kept);
        };
        const auto store = [&](auto& batch, int i) {
          batch.store(out + i * V + e, V, e & 7, keep_of, t, ch, live, kept);
        };
        // the next rows are on their way while these are worked on
        Batch<T, W, kRows, MASK, IN_PLACE> one, two;
        if (i + kRows <= row_last) load(one, i);
        while (i + kRows <= row_last) {
          if (i + step + kRows <= row_last) load(two, i + step);
          store(one, i);
          i += step;
          if (i + kRows > row_last) break;
          if (i + step + kRows <= row_last) load(one, i + step);
          store(two, i);
          i += step;
        }
        for (const int last = min(i + kRows, row_last); i < last; ++i) {
          Batch<T, W, 1, MASK, IN_PLACE> rest;
          load(rest, i);
          store(rest, i);
        }
      });
    }
  }
  if (!tree) return;
  __syncthreads();

  // the tree's tokens: each row by its own path's count
  for (int j = tid; j < (row_last - row_first) * owns; j += kThreads) {
    const int i = row_first + j / owns, m = j % owns, e = own_token[m];
    float y = to_f32(logits[i * V + e]);
    if (MASK && !(mask[(size_t)i * mask_words + ((c0 + e) >> 5)] >> ((c0 + e) & 31) & 1)) continue;
    const uint32_t base = counts[e];
    const int mine = __popcll(own_nodes[m] & path[i]);
    const uint32_t c = (base & ~kPrompt) + mine;
    if (base != 0 || mine) y *= y > 0.f ? tables.rep_inv : rep;
    if (c) y -= freq * (float)c + pres;
    out[i * V + e] = from_f32<T>(y + tables.bias_of(e));
  }
}

namespace {

using Kernel = void (*)(TreeLogitsParams, int, int, int, bool);

template <typename T, int W, bool MASK, bool IN_PLACE>
Kernel kernel_of(const TreeLogitsParams& p) {
  if constexpr (W > 0) {
    if (p.N < kRowsOf<T>) return tree_logits_kernel<T, W, MASK, IN_PLACE, true>;
  }
  return tree_logits_kernel<T, W, MASK, IN_PLACE, false>;
}

template <typename T, int W>
Kernel kernel_of(const TreeLogitsParams& p) {
  if (p.logits == p.out)
    return p.mask ? kernel_of<T, W, true, true>(p) : kernel_of<T, W, false, true>(p);
  return p.mask ? kernel_of<T, W, true, false>(p) : kernel_of<T, W, false, false>(p);
}

template <typename T>
Kernel kernel_of(const TreeLogitsParams& p) {
  const uintptr_t all = (uintptr_t)p.logits | (uintptr_t)p.out | (uintptr_t)p.V * sizeof(T);
  if (all % 16 == 0) return kernel_of<T, 16>(p);
  if constexpr (sizeof(T) == 4) return kernel_of<T, 4>(p);
  else return all % 8 == 0 ? kernel_of<T, 8>(p) : kernel_of<T, 0>(p);
}

}  // namespace

template <typename T>
cudaError_t launch_tree_logits_of(const TreeLogitsParams& p, int num_sms, cudaStream_t stream) {
  // One wave of CTAs, if chunks of 512 to 32768 tokens allow it: a history is counted once per chunk.
  // Counts of 16 bits only where those of 32 need more memory than the wave leaves (64 x 1 over 128000:
  // 24 us with three CTAs an SM, 28 with two): they cost a shift each.
  const auto smem_of = [&](int chunk, bool narrow) {
    const int biases = p.bias_token ? p.max_bias < chunk ? p.max_bias : chunk : 0;
    return (at(narrow ? chunk / 2 : chunk) + 4 * (chunk / 32 + 1) + 3 + biases + 3) / 4 * 16;
  };
  constexpr int kOwn = 7168;  // static shared memory and what the system keeps
  int chunks = 0, chunk = 0, slots = 0;
  bool narrow = false;
  for (int per_sm = kCtas; per_sm > 0; --per_sm) {
    slots = per_sm * num_sms;
    chunks = slots / p.R < 1 ? 1 : slots / p.R;
    const int most = (p.V + 511) / 512;
    chunks = chunks > most ? most : chunks;
    chunk = ((p.V + chunks - 1) / chunks + 255) / 256 * 256;
    chunk = chunk > 32768 ? 32768 : chunk;
    const int room = (228 << 10) / per_sm - kOwn;
    narrow = smem_of(chunk, false) > room && p.H <= kNarrow;
    if (smem_of(chunk, narrow) <= room) break;
  }
  while (smem_of(chunk, narrow) > kSmemMost) chunk /= 2;
  chunks = (p.V + chunk - 1) / chunk;
  int parts = 1;
  while (parts * 8 <= p.N && (int64_t)p.R * chunks * parts * 2 <= slots) parts *= 2;
  if ((int64_t)p.R * parts * chunks > INT32_MAX) return cudaErrorInvalidConfiguration;
  const int smem = smem_of(chunk, narrow);
  const unsigned grid = (unsigned)p.R * parts * chunks;
  const Kernel kernel = kernel_of<T>(p);
  if (smem > (40 << 10)) {  // with the static part, more than a launch has by itself
    // always the same limit: another thread's call may come between this one and the launch
    const cudaError_t e =
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMost);
    if (e != cudaSuccess) return e;
  }
  kernel<<<grid, kThreads, smem, stream>>>(p, chunk, chunks, parts, narrow);
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace flare
