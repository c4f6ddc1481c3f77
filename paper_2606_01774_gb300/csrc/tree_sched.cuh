// How the softmax attention of a batch of drafted trees is spread over the GPU.
//
// A request with a prefix of P tokens has n = ceil(P / 64) + 1 key tiles per
// kv head: its prefix, 64 tokens a tile, and one tile with its nodes' own keys
// (at most 64).  The tiles of the whole batch, in the order (request, kv head,
// tile), are cut into `gangs` spans of equal length; a gang has one CTA per
// tile of query rows, and each walks the gang's span for its own rows, so the
// row tiles read a key tile at about the same time and it leaves DRAM once.
// Equal spans load every SM alike whether the batch is one long prefix or many
// ragged ones.  Where a span ends inside a (request, kv head) item, the item's
// pieces are merged afterwards from partial outputs in a fixed order.  A CTA
// has at most two partial pieces: slot 0, one that starts inside an item (its
// first), and slot 1, one that starts an item without finishing it (its last).
//
// Lengths live on the device, so every CTA computes the cut itself.  Whether a
// request's pages and tree are sound does not enter it: that is checked beside
// the attention, and a bad request's pieces are dropped where they would be
// stored.
#pragma once

#include "common.cuh"
#include "kernels.h"

namespace flare {

constexpr int kTreeTile = 64;  // keys per tile
// Pieces of an item that its last piece merges itself (bf16).  More of them,
// or a prefix over the whole GPU, leave few CTAs to read many partials:
// tree_finish_kernel takes those.
constexpr int kTreeJoin = 4;

// The query rows of row tile `tile` of a (request, kv head) item: whole nodes
// with their G query heads, or, with more heads than a tile has rows, some of
// one node's heads.  Row i is head head0 + i % heads of node node0 + i / heads.
struct TreeRows {
  int node0, nodes, head0, heads;
  __device__ __forceinline__ int node(int i) const { return node0 + i / heads; }
  __device__ __forceinline__ int head(int i) const { return head0 + i % heads; }
  // whether row i is one, of a tree of n nodes
  __device__ __forceinline__ bool used(int i, int n) const {
    return i < nodes * heads && node(i) < n;
  }
};

__device__ __forceinline__ TreeRows tree_rows(const TreeSoftmaxParams& p, int tile) {
  if (p.G <= p.tile_base) {
    const int nodes = p.tile_base / p.G;
    return TreeRows{tile * nodes, nodes, 0, p.G};
  }
  const int per = (p.G + p.tile_base - 1) / p.tile_base;  // tiles per node
  const int h = tile % per * p.tile_base;
  return TreeRows{tile / per, 1, h, min(p.tile_base, p.G - h)};
}

// An item that a gang starts and leaves unfinished, for tree_finish_kernel: its
// request and kv head, and the first and last gang that have a piece of it.
struct alignas(16) TreeCut {
  int r, kvh, nodes, first, last;
};

// Key tiles per kv head of a request; 0 when it has no nodes or a wrong length.
__device__ __forceinline__ int tree_tiles(const TreeSoftmaxParams& p, int r) {
  const int n = p.node_len[r], P = p.prefix_len[r];
  const bool ok = n > 0 && n <= p.N && P >= 0 && P <= (long long)p.max_pages * p.page_size;
  return ok ? (P + kTreeTile - 1) / kTreeTile + 1 : 0;
}

// A stretch of one item's tiles: j0 .. j1 - 1 of n.
struct TreePiece {
  int r, kvh, j0, j1, n;
  __device__ bool whole() const { return j0 == 0 && j1 == n; }
  __device__ int slot() const { return j0 == 0 ? 1 : 0; }
};

struct TreeCursor {
  int r, kvh, j;
  long long left;

  // The next piece of the span; false at its end.
  __device__ __forceinline__ bool next(const TreeSoftmaxParams& p, TreePiece& w) {
    if (left <= 0) return false;
    int n = tree_tiles(p, r);
    while (n == 0) n = tree_tiles(p, ++r);
    w.r = r;
    w.kvh = kvh;
    w.j0 = j;
    w.j1 = (int)(left < n - j ? j + left : n);
    w.n = n;
    left -= w.j1 - w.j0;
    if (w.j1 == n) {
      j = 0;
      if (++kvh == p.Hkv) {
        kvh = 0;
        ++r;
      }
    } else {
      j = w.j1;
    }
    return true;
  }
};

// How many of the plan's gangs have work: each of them at least a tile.
__device__ __forceinline__ int tree_gangs(const TreeSoftmaxParams& p, long long total) {
  return total < p.gangs ? (int)total : p.gangs;
}

// First row of a CTA's partial outputs for its piece of an item that gang g0
// starts: g0's own is its last piece (slot 1), the others' their first.
__device__ __forceinline__ size_t tree_part(const TreeSoftmaxParams& p, int g, int g0, int mt) {
  return (((size_t)g * p.row_tiles + mt) * 2 + (g == g0 ? 1 : 0)) * p.tile_rows;
}
// Columns 4 c4 .. 4 c4 + 3 of row `row` of the partial output whose first row
// is `part`: rows run fastest, since it is written and read by a thread per row.
__device__ __forceinline__ float4* tree_part_at(const TreeSoftmaxParams& p, size_t part, int row,
                                                int c4) {
  return reinterpret_cast<float4*>(p.part_o + part * p.D) + (size_t)c4 * p.tile_rows + row;
}

// a / b of non-negative numbers: in 32 bits where both fit, a fifth of the time.
__device__ __forceinline__ long long tree_div(long long a, long long b) {
  return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}

// The gang whose span holds tile x of `total`.
__device__ __forceinline__ int tree_gang_of(long long x, long long total, int gangs) {
  return (int)tree_div((x + 1) * gangs - 1, total);
}

__device__ __forceinline__ long long shfl_up_ll(long long x, int o) {
  return __shfl_up_sync(0xffffffffu, x, o);
}

// The batch's cut and one gang's span, [lo, hi) of `total` tiles, by a warp on
// its own (every warp of a CTA works it out for itself: that takes one round
// trip to memory and no barrier).
struct TreeSpan {
  long long lo, hi, total;
  int gangs;
  TreeCursor start;
};

__device__ __forceinline__ TreeSpan tree_span(const TreeSoftmaxParams& p, int gang) {
  const int lane = threadIdx.x & 31;
  const int per = (p.R + 31) / 32;
  const int r0 = min(p.R, lane * per), r1 = min(p.R, r0 + per);
  long long sum = 0;
#pragma unroll 4
  for (int r = r0; r < r1; ++r) sum += (long long)tree_tiles(p, r) * p.Hkv;
  long long incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = shfl_up_ll(incl, o);
    if (lane >= o) incl += x;
  }
  TreeSpan s;
  s.total = __shfl_sync(0xffffffffu, incl, 31);
  s.gangs = tree_gangs(p, s.total);
  s.lo = s.hi = 0;
  if (gang < s.gangs) {
    s.lo = tree_div(s.total * gang, s.gangs);
    s.hi = tree_div(s.total * (gang + 1), s.gangs);
  }
  s.start.left = s.hi - s.lo;
  s.start.r = s.start.kvh = s.start.j = 0;
  if (s.lo == s.hi) return s;
  // the lane that holds the first request walks to it
  const bool mine = incl - sum <= s.lo && s.lo < incl;
  if (mine) {
    long long at = s.lo - (incl - sum);
    int r = r0, n = tree_tiles(p, r);
    while (at >= (long long)n * p.Hkv) {
      at -= (long long)n * p.Hkv;
      n = tree_tiles(p, ++r);
    }
    s.start.r = r;
    s.start.kvh = (int)tree_div(at, n);
    s.start.j = (int)(at - (long long)s.start.kvh * n);
  }
  const int src = __ffs(__ballot_sync(0xffffffffu, mine)) - 1;
  s.start.r = __shfl_sync(0xffffffffu, s.start.r, src);
  s.start.kvh = __shfl_sync(0xffffffffu, s.start.kvh, src);
  s.start.j = __shfl_sync(0xffffffffu, s.start.j, src);
  return s;
}

// The first and last gang that have a piece of piece w's item: it starts j0
// tiles before the span, or ends with it.
__device__ __forceinline__ void tree_sharers(const TreeSpan& s, const TreePiece& w, int& g0,
                                             int& g1) {
  const long long s0 = w.slot() ? s.hi - w.j1 : s.lo - w.j0;
  g0 = tree_gang_of(s0, s.total, s.gangs);
  g1 = tree_gang_of(s0 + w.n - 1, s.total, s.gangs);
}

// Puts the item that a gang starts and does not finish on the list of those
// that tree_finish_kernel merges (its order does not matter).  One thread of the
// gang's first CTA, with each of its pieces, after the plan has emptied the list.
__device__ __forceinline__ void tree_list_cut(const TreeSoftmaxParams& p, const TreeSpan& s,
                                              const TreePiece& w) {
  if (w.whole() || w.slot() == 0) return;
  int g0, g1;
  tree_sharers(s, w, g0, g1);
  if (g1 - g0 < p.join) return;
  static_cast<TreeCut*>(p.cuts)[atomicAdd(p.n_cuts, 1)] =
      TreeCut{w.r, w.kvh, p.node_len[w.r], g0, g1};
}

}  // namespace flare
