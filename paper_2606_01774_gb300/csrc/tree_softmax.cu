// Softmax attention of drafted trees over a paged KV prefix: the kernels
// around the attention itself (tree_sched.cuh has how the work is cut), and
// the fp32 attention kernel on CUDA cores.
//
//   tree_plan_kernel    a CTA per request checks its lengths, page ids and
//                       tree, and writes its nodes' paths
//   attention           bf16: tree_softmax_tc.cu; fp32: tree_softmax_simt_kernel
//   tree_finish_kernel  merges items that several gangs share, and writes the
//                       outputs of unused nodes
// Each starts while the one before it runs (pdl.cuh) and waits for it where it
// needs its results.
//
// Online softmax in base 2 with the logit scale folded into q; running
// maximum, sum and output in fp32.
#include <limits>

#include "async.cuh"
#include "common.cuh"
#include "kernels.h"
#include "pdl.cuh"
#include "tree.cuh"
#include "tree_sched.cuh"

namespace flare {

namespace {

constexpr int kPlanThreads = 128;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ void store4(float* x, float4 v) { *reinterpret_cast<float4*>(x) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* x, float4 v) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(x) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo),
                                            *reinterpret_cast<const uint32_t*>(&hi));
}

// CTAs per SM of the fp32 kernel: its shared memory, and registers for 16 warps
__host__ __device__ constexpr int simt_ctas(int D, int rows) {
  return rows == 32 ? 256 / D : D == 64 ? 2 : 1;
}

}  // namespace

__global__ void __launch_bounds__(kPlanThreads) tree_plan_kernel(TreeSoftmaxParams p) {
  pdl_launch_next();
  const int r = blockIdx.x, tid = threadIdx.x;
  for (int i = r * kPlanThreads + tid; i < p.n_counts; i += gridDim.x * kPlanThreads)
    p.counts[i] = 0;
  if (r == 0 && tid == 0) *p.n_cuts = 0;
  const int n = p.node_len[r], P = p.prefix_len[r];
  int bad = 0;
  if (n < 0 || n > p.N) bad |= FLARE_DEV_BAD_TREE;
  if (P < 0 || P > (long long)p.max_pages * p.page_size) bad |= FLARE_DEV_BAD_PREFIX_LEN;
  if (!bad && n > 0) {
    const int pages = (P + p.page_size - 1) / p.page_size;
    for (int i = tid; i < pages; i += kPlanThreads) {
      const int pg = p.page_table[(size_t)r * p.max_pages + i];
      if (pg < 0 || pg >= p.num_pages) bad |= FLARE_DEV_BAD_PAGE;
    }
    if (tid < 32) {
      int p0, p1;
      if (warp_load_tree(p.parent + (size_t)r * p.N, n, p0, p1)) {
        uint64_t a0, a1;
        warp_paths(n, p0, p1, a0, a1);
        if (tid < p.N) p.anc[(size_t)r * p.N + tid] = a0;
        if (tid + 32 < p.N) p.anc[(size_t)r * p.N + tid + 32] = a1;
      } else {
        bad |= FLARE_DEV_BAD_TREE;
      }
    }
  }
  const int any = __syncthreads_or(bad);
  if (bad) flag(p.dev_status, bad);
  if (tid == 0) p.bad[r] = any;
}

// fp32 attention.  A CTA takes ROWS = 32 or 64 query rows; thread (y, x) of its
// ROWS / 4 x 16 holds rows 4y .. 4y+3 against keys x, x+16, x+32, x+48 of a tile,
// and columns 4x (+ 64 c) of those rows' outputs, in packed pairs: of dimensions in
// the scores, of columns in the output.  Bound by shared memory's 16-byte reads (one
// per four packed multiply-adds) and the multiply-adds (4 D per row and key against
// 8 D bytes per key).  Copies run a tile ahead, keys while the previous tile's values
// are at work and values under the next scores (staged between the products, the same
// calls took about twice as long).  The whole call, prefixes of 1150 tokens: 48
// requests x 61 nodes, D = 64 235 us (31 TFLOP/s of 74); 32 x 16 nodes, D = 128 158
// us; 16 x 16 nodes, D = 256 160 us; 12 x 13 nodes, prefixes below 1022, D = 64 21 us,
// a latency of three launches and one tile.
template <int D, int ROWS>
__global__ void __launch_bounds__(4 * ROWS, simt_ctas(D, ROWS))
    tree_softmax_simt_kernel(TreeSoftmaxParams p) {
  constexpr int kThreadsS = 4 * ROWS;
  constexpr int kS = D + 4;  // row stride of staged rows: 16 lanes on 16 rows spread over the banks
  constexpr int kC = D / 64;
  extern __shared__ __align__(16) float sm[];
  float* Qs = sm;                    // [ROWS][kS]
  float* Ks = Qs + ROWS * kS;      // [64][kS]
  float* Vs = Ks + kTreeTile * kS;   // [64][kS]
  float* Ps = Vs + kTreeTile * kS;   // [ROWS][64 + 4]
  constexpr int kPS = kTreeTile + 4;
  __shared__ size_t row_at[kTreeTile];

  const int tid = threadIdx.x, x = tid & 15, y = tid >> 4;
  const int gang = blockIdx.x / p.row_tiles, mt = blockIdx.x % p.row_tiles;
  const TreeRows rows = tree_rows(p, mt);
  const float* q = static_cast<const float*>(p.q);
  const float* pools[2] = {static_cast<const float*>(p.k_pool), static_cast<const float*>(p.v_pool)};
  const float* blks[2] = {static_cast<const float*>(p.k_blk), static_cast<const float*>(p.v_blk)};
  const TreeSpan span = tree_span(p, gang);
  TreeCursor cur = span.start;
  auto next_piece = [&](TreePiece& w) {
    while (cur.next(p, w))
      if (rows.node0 < p.node_len[w.r]) return true;
    return false;
  };
  // where a tile's rows are: page ids asked for first (find), offsets later
  // (locate; ~0: none), by a thread per row; then copies, zeros for no row
  auto find = [&](const TreePiece& w, int j) {
    const int tok = j * kTreeTile + tid;
    return tid < kTreeTile && j < w.n - 1 && tok < p.prefix_len[w.r]
               ? p.page_table[(size_t)w.r * p.max_pages + tok / p.page_size]
               : -1;
  };
  auto locate = [&](const TreePiece& w, int j, int page) {
    if (tid >= kTreeTile) return;
    size_t at = ~(size_t)0;
    if (j == w.n - 1) {
      if (tid < p.node_len[w.r]) at = (((size_t)w.r * p.N + tid) * p.Hkv + w.kvh) * D;
    } else if (page >= 0 && page < p.num_pages) {  // the plan may not be through yet
      at = (((size_t)page * p.Hkv + w.kvh) * p.page_size + (j * kTreeTile + tid) % p.page_size) * D;
    }
    row_at[tid] = at;
  };
  auto stage = [&](float* dst, int kv, bool tree) {
    const float* src = (tree ? blks[kv] : pools[kv]) + tid % (D / 4) * 4;
    dst += tid % (D / 4) * 4;
#pragma unroll 4
    for (int i = tid / (D / 4); i < kTreeTile; i += kThreadsS / (D / 4)) {
      const size_t at = row_at[i];
      const bool live = at != ~(size_t)0;
      cp_async16(dst + i * kS, src + (live ? at : 0), live);
    }
    cp_async_commit();
  };
  TreePiece w, nx;
  bool more = next_piece(w), planned = false;
  if (more) {
    locate(w, w.j0, find(w, w.j0));
    __syncthreads();
    stage(Ks, 0, w.j0 == w.n - 1);
    stage(Vs, 1, w.j0 == w.n - 1);
  }
  for (; more; w = nx) {
    more = next_piece(nx);
    const int n = p.node_len[w.r], P = p.prefix_len[w.r];
    for (int e = tid; e < ROWS * (D / 4); e += kThreadsS) {
      const int i = e / (D / 4), d = e % (D / 4) * 4;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (rows.used(i, n))
        v = *reinterpret_cast<const float4*>(
            q + (((size_t)w.r * p.N + rows.node(i)) * p.Hq + w.kvh * p.G + rows.head(i)) * D + d);
      *reinterpret_cast<float4*>(Qs + i * kS + d) =
          make_float4(v.x * p.scale_log2, v.y * p.scale_log2, v.z * p.scale_log2, v.w * p.scale_log2);
    }
    if (!planned) {
      pdl_wait();  // the plan
      pdl_launch_next();
      planned = true;
    }
    if (mt == 0 && tid == 0) tree_list_cut(p, span, w);
    uint64_t path[4];  // the keys of the tree tile that each row sees
    bool mine = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * y + i;
      const bool used = rows.used(row, n);
      path[i] = used ? p.anc[(size_t)w.r * p.N + rows.node(row)] : 0ull;
      mine = mine || used;
    }
    const bool warp_live = __any_sync(0xffffffffu, mine);  // else it copies only
    uint64_t acc[4][2 * kC];  // pairs of columns
    float mrow[4], lrow[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      mrow[i] = -INFINITY;
      lrow[i] = 0.f;
#pragma unroll
      for (int c = 0; c < 2 * kC; ++c) acc[i][c] = 0ull;
    }
    for (int j = w.j0; j < w.j1; ++j) {
      const bool tree = j == w.n - 1;
      const int valid = min(kTreeTile, P - j * kTreeTile);  // of a prefix tile
      const bool last = j + 1 == w.j1, load = !last || more;  // another tile follows
      const TreePiece& then = last ? nx : w;
      const int jn = last ? nx.j0 : j + 1, page = load ? find(then, jn) : -1;
      cp_async_wait<1>();
      __syncthreads();  // the keys (and a piece's queries)
      uint64_t s2[4][4];  // even and odd dimensions' sums
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) s2[i][c] = 0ull;
#pragma unroll 4
      for (int d = 0; d < (warp_live ? D : 0); d += 4) {
        ulonglong2 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          a[i] = *reinterpret_cast<const ulonglong2*>(Qs + (4 * y + i) * kS + d);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          b[c] = *reinterpret_cast<const ulonglong2*>(Ks + (x + 16 * c) * kS + d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            s2[i][c] = f2_fma(a[i].y, b[c].y, f2_fma(a[i].x, b[c].x, s2[i][c]));
      }
      if (load) locate(then, jn, page);
      __syncthreads();  // the keys are read
      if (load) stage(Ks, 0, jn == then.n - 1);
      if (warp_live) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float s[4], mx = -INFINITY;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float even, odd;
            f2_split(s2[i][c], even, odd);
            const int key = x + 16 * c;
            const bool see = tree ? (path[i] >> key) & 1 : key < valid;
            s[c] = see ? even + odd : -INFINITY;
            mx = fmaxf(mx, s[c]);
          }
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
          const float mnew = fmaxf(mrow[i], mx);
          const float mref = mnew == -INFINITY ? 0.f : mnew;  // a row that sees nothing yet
          const float corr = exp2f(mrow[i] - mref);
          float sum = 0.f;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float e = exp2f(s[c] - mref);
            Ps[(4 * y + i) * kPS + x + 16 * c] = e;
            sum += e;
          }
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          lrow[i] = lrow[i] * corr + sum;
          mrow[i] = mnew;
#pragma unroll
          for (int c = 0; c < 2 * kC; ++c) acc[i][c] = f2_mul(f2_dup(corr), acc[i][c]);
        }
      }
      if (load) cp_async_wait<1>();
      else cp_async_wait<0>();
      __syncthreads();  // the values (a row's probabilities come from its own warp)
#pragma unroll 1
      for (int k = 0; k < (warp_live ? kTreeTile : 0); k += 4) {
        float4 pr[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          pr[i] = *reinterpret_cast<const float4*>(Ps + (4 * y + i) * kPS + k);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
          for (int c = 0; c < kC; ++c) {
            const ulonglong2 v =
                *reinterpret_cast<const ulonglong2*>(Vs + (k + kk) * kS + 4 * x + 64 * c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float pk = kk == 0 ? pr[i].x : kk == 1 ? pr[i].y : kk == 2 ? pr[i].z : pr[i].w;
              acc[i][2 * c] = f2_fma(f2_dup(pk), v.x, acc[i][2 * c]);
              acc[i][2 * c + 1] = f2_fma(f2_dup(pk), v.y, acc[i][2 * c + 1]);
            }
          }
      }
      __syncthreads();  // the values are read
      if (load) stage(Vs, 1, jn == then.n - 1);
    }
    if (p.bad[w.r]) continue;
    const bool whole = w.whole();
    const size_t part = ((size_t)blockIdx.x * 2 + w.slot()) * ROWS;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * y + i;
      if (!rows.used(row, n)) continue;
      const float inv = lrow[i] > 0.f ? 1.f / lrow[i] : 0.f;
      const float l2 = lrow[i] > 0.f ? mrow[i] + log2f(lrow[i]) : -INFINITY;
      const size_t o =
          ((size_t)w.r * p.N + rows.node(row)) * p.Hq + w.kvh * p.G + rows.head(row);
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        float4 a;
        f2_split(f2_mul(f2_dup(inv), acc[i][2 * c]), a.x, a.y);
        f2_split(f2_mul(f2_dup(inv), acc[i][2 * c + 1]), a.z, a.w);
        if (whole) store4(static_cast<float*>(p.out) + o * D + 4 * x + 64 * c, a);
        else *tree_part_at(p, part, row, x + 16 * c) = a;
      }
      if (x == 0) {
        if (!whole) p.part_lse[part + row] = l2;
        else if (p.lse) p.lse[o] = l2 * kLn2;
      }
    }
  }
  if (!planned) {
    pdl_wait();
    pdl_launch_next();
  }
}

// Writes the unused nodes' rows, and merges the items that the attention left
// in pieces (more than p.join of them), in gang order, whatever the timing:
//     out = sum_s 2^(lse_s - lse) out_s.
// A thread takes four columns of a row; PARTS threads share them, each with
// every PARTS-th piece: one, or eight, where rows are few and may have many
// pieces.
template <typename T, int D, int PARTS>
__global__ void __launch_bounds__(256) tree_finish_kernel(TreeSoftmaxParams p) {
  constexpr int kPer = 256 / PARTS;  // (row, column group) elements per CTA and pass
  constexpr int kIn = PARTS > 1 ? 10 : 4;  // pieces in flight per thread
  __shared__ float4 red_o[PARTS > 1 ? 256 : 1];
  __shared__ float2 red_l[PARTS > 1 ? 256 : 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // unused nodes' rows, a node per warp (the attention kernel waited for the
  // plan before it let this one start)
  for (long long u = (long long)blockIdx.x * 8 + warp; u < (long long)p.R * p.N;
       u += (long long)gridDim.x * 8) {
    const int r = (int)(u / p.N), t = (int)(u - (long long)r * p.N);
    if (p.bad[r] || t < p.node_len[r]) continue;
    uint4* out = reinterpret_cast<uint4*>(static_cast<T*>(p.out) + u * p.Hq * D);
    const int n16 = p.Hq * (D * (int)sizeof(T) / 16);
    for (int e = lane; e < n16; e += 32) out[e] = make_uint4(0u, 0u, 0u, 0u);
    if (p.lse)
      for (int e = lane; e < p.Hq; e += 32) p.lse[u * p.Hq + e] = -INFINITY;
  }
  pdl_wait();  // the attention
  // rows that may be used, rounded up so that elements split by shifts
  const int used = p.N * p.G < p.tile_rows ? p.N * p.G : p.tile_rows;
  int shift = 0;
  while ((1 << shift) < used) ++shift;
  const int passes = ((D / 4 << shift) + kPer - 1) / kPer;
  // both in one round trip: the list's length, and the first unit's entry (the
  // list has room for every gang's)
  const long long units = (long long)*p.n_cuts * p.row_tiles * passes;
  const TreeCut* cuts = static_cast<const TreeCut*>(p.cuts);
  TreeCut cut = cuts[min(blockIdx.x / (passes * p.row_tiles), p.gangs - 1)];
  for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int at = (int)(unit / passes), e = (int)(unit - (long long)at * passes) * kPer + tid % kPer;
    if (unit != blockIdx.x) cut = cuts[at / p.row_tiles];
    const int g0 = cut.first, mt = at % p.row_tiles;
    const int row = e & ((1 << shift) - 1), c4 = e >> shift, sub = tid / kPer;
    const bool skip = p.bad[cut.r] != 0;
    const TreeRows rows = tree_rows(p, mt * (p.tile_rows / p.tile_base) + row / p.tile_base);
    const int i = row % p.tile_base;
    const bool live = c4 < D / 4 && row < p.tile_rows && rows.used(i, cut.nodes);
    // this thread's pieces: running maximum, sum of weights, weighted output
    float mx = -INFINITY, den = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    auto take = [&](float l, float d, float4 x) {
      if (l == -INFINITY) return;  // the row sees nothing of it
      const float mn = fmaxf(mx, l), corr = exp2f(mx - mn), f = exp2f(l - mn);
      den = den * corr + f * d;
      mx = mn;
      acc.x = fmaf(f, x.x, acc.x * corr);
      acc.y = fmaf(f, x.y, acc.y * corr);
      acc.z = fmaf(f, x.z, acc.z * corr);
      acc.w = fmaf(f, x.w, acc.w * corr);
    };
    if (live) {
      for (int g = g0 + sub; g <= cut.last; g += PARTS * kIn) {
        float l[kIn];
        float4 x[kIn];
#pragma unroll
        for (int u = 0; u < kIn; ++u) {
          const int gg = g + u * PARTS;
          const size_t part = tree_part(p, gg, g0, mt);
          l[u] = gg <= cut.last ? p.part_lse[part + row] : -INFINITY;
          x[u] = gg <= cut.last ? *tree_part_at(p, part, row, c4) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int u = 0; u < kIn; ++u) take(l[u], 1.f, x[u]);
      }
    }
    if constexpr (PARTS > 1) {
      __syncthreads();  // the previous unit's are read
      red_o[tid] = acc;
      red_l[tid] = make_float2(mx, den);
      __syncthreads();
      if (sub != 0) continue;
#pragma unroll
      for (int u = 1; u < PARTS; ++u)
        take(red_l[u * kPer + tid].x, red_l[u * kPer + tid].y, red_o[u * kPer + tid]);
    }
    if (!live || skip) continue;
    const size_t o = ((size_t)cut.r * p.N + rows.node(i)) * p.Hq + cut.kvh * p.G + rows.head(i);
    const float inv = den > 0.f ? 1.f / den : 0.f;
    store4(static_cast<T*>(p.out) + o * D + 4 * c4,
           make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
    if (c4 == 0 && p.lse) p.lse[o] = den > 0.f ? (mx + log2f(den)) * kLn2 : -INFINITY;
  }
}

TreeSoftmaxPlan plan_tree_softmax(int R, int N, int Hq, int Hkv, int D, int page_size,
                                  int max_pages, bool bf16, int num_sms) {
  TreeSoftmaxPlan pl;
  const int G = Hq / Hkv;
  // fp32: row tiles of 64 where one of 32 does not hold all rows (64 rows over 1150
  // tokens: 16 requests, D = 256 210 -> 167 us, 32 requests, D = 128 180 -> 172 us)
  pl.tile_base = bf16 ? 128 : (long long)N * G > 32 ? 64 : 32;
  const int per_node = G <= pl.tile_base ? 1 : (G + pl.tile_base - 1) / pl.tile_base;
  const int nodes = G <= pl.tile_base ? pl.tile_base / G : 1;  // of a row tile
  const long long tiles = (N + nodes - 1) / nodes * (long long)per_node;
  // bf16: two row tiles share a CTA's keys where there are two and tensor
  // memory holds both (D <= 128).  96 requests of 61 nodes, 244 rows, D = 128:
  // 127 us where one row tile a CTA took 150 us when this came in (85 us by now).
  const int per_cta = bf16 && D <= 128 && tiles > 1 ? 2 : 1;
  pl.tile_rows = per_cta * pl.tile_base;
  pl.row_tiles = (int)((tiles + per_cta - 1) / per_cta);
  const int per_sm = bf16 ? 1 : simt_ctas(D, pl.tile_base);
  // as many gangs as the GPU holds at once, and no more than there can be tiles
  long long gangs = (long long)num_sms * per_sm / pl.row_tiles;
  const long long most =
      (long long)R * Hkv * (((long long)max_pages * page_size + kTreeTile - 1) / kTreeTile + 1);
  if (gangs > most) gangs = most;
  if (gangs < 1) gangs = 1;
  pl.gangs = (int)gangs;
  const size_t slots = (size_t)2 * pl.gangs * pl.row_tiles * pl.tile_rows;
  pl.join = bf16 ? kTreeJoin : 0;
  pl.n_counts = bf16 ? pl.gangs * pl.row_tiles * (pl.tile_rows / pl.tile_base) : 0;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  size_t at = 0;
  pl.bad_off = at;
  at += up((size_t)R * sizeof(int32_t));
  pl.n_cuts_off = at;
  at += up(sizeof(int32_t));
  pl.cuts_off = at;
  at += up((size_t)pl.gangs * sizeof(TreeCut));
  pl.counts_off = at;
  at += up((size_t)pl.n_counts * sizeof(int32_t));
  pl.anc_off = at;
  at += up((size_t)R * N * sizeof(uint64_t));
  pl.part_o_off = at;
  at += up(slots * D * sizeof(float));
  pl.part_lse_off = at;
  at += up(slots * sizeof(float));
  pl.workspace_bytes = at;
  return pl;
}

namespace {

template <int D, int ROWS>
cudaError_t launch_simt_rows(const TreeSoftmaxParams& p, cudaStream_t stream) {
  const int smem =
      (int)sizeof(float) * ((ROWS + 2 * kTreeTile) * (D + 4) + ROWS * (kTreeTile + 4));
  cudaError_t e = cudaFuncSetAttribute(tree_softmax_simt_kernel<D, ROWS>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  e = pdl_launch(tree_softmax_simt_kernel<D, ROWS>, dim3((unsigned)(p.gangs * p.row_tiles)),
                 4 * ROWS, smem, stream, true, 1, p);
  note_launches(1);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <int D>
cudaError_t launch_simt_d(const TreeSoftmaxParams& p, cudaStream_t stream) {
  return p.tile_base == 64 ? launch_simt_rows<D, 64>(p, stream) : launch_simt_rows<D, 32>(p, stream);
}

template <typename T, int D>
cudaError_t launch_finish(const TreeSoftmaxParams& p, cudaStream_t stream) {
  const dim3 grid(4 * kNumSMs);
  const cudaError_t e =
      (long long)p.N * p.G <= 16
          ? pdl_launch(tree_finish_kernel<T, D, 8>, grid, 256, 0, stream, true, 1, p)
          : pdl_launch(tree_finish_kernel<T, D, 1>, grid, 256, 0, stream, true, 1, p);
  note_launches(1);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <int D>
cudaError_t launch_d(const TreeSoftmaxParams& p, bool bf16, cudaStream_t stream) {
  // everything the host has to prepare comes first, the three launches in a row
  TreeSoftmaxTc tc;
  if (bf16) {
    const cudaError_t e = prepare_tree_softmax_tc(p, &tc);
    if (e != cudaSuccess) return e;
  }
  tree_plan_kernel<<<(unsigned)p.R, kPlanThreads, 0, stream>>>(p);
  note_launches(1);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  e = bf16 ? launch_tree_softmax_tc(p, tc, stream) : launch_simt_d<D>(p, stream);
  if (e != cudaSuccess) return e;
  return bf16 ? launch_finish<__nv_bfloat16, D>(p, stream) : launch_finish<float, D>(p, stream);
}

}  // namespace

cudaError_t launch_tree_softmax(const TreeSoftmaxParams& params, bool bf16, cudaStream_t stream) {
  TreeSoftmaxParams p = params;
  // The bf16 kernel masks scores by -inf before it scales them, which 0 would turn
  // into a NaN.  The least positive float instead leaves a score below 2^126 less than
  // 2^-23 of a weight, and -inf as it is.
  if (bf16 && p.scale_log2 == 0.f) p.scale_log2 = std::numeric_limits<float>::denorm_min();
  switch (p.D) {
    case 64: return launch_d<64>(p, bf16, stream);
    case 128: return launch_d<128>(p, bf16, stream);
    case 256: return launch_d<256>(p, bf16, stream);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace flare
