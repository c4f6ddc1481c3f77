// Softmax attention of drafted trees over a paged KV prefix on the
// 5th-generation tensor cores (tcgen05), bf16 in, fp32 accumulate.
//
// tree_sched.cuh has how the work is cut: a CTA walks its gang's span of key
// tiles for its own row tiles of 128 query rows (the nodes' queries of one kv
// head's G query heads, which share its keys).  A piece is a stretch of one
// item's tiles: prefix tiles through the page table, 64 tokens each, and the
// item's last tile, the tree's own keys, masked by the rows' path bits.  A
// piece that covers its item stores the output.  Of an item in up to kTreeJoin
// pieces the one that ends last takes the others' partial outputs in, its own
// still in tensor memory (in gang order, whichever it is); the pieces of longer
// items are merged by tree_finish_kernel, over more of the GPU.
//
// Serving trees are bound by the keys' and values' bytes: a tile of 64 keys is
// 256 D bytes for 4 x 128 x 64 D operations, which the tensor cores finish in a
// third of the time that its share of DRAM bandwidth gives it, padded rows and
// all.  So the kernel is built as a stream: queries in shared memory, rings of
// TMA boxes in the rest of it (a tile takes about a microsecond from issue to
// arrival), scores, probabilities and output in tensor memory, and a persistent
// CTA that keeps the rings full across pieces.
//
// NQ = 2 (more than one row tile, D <= 128): two row tiles with a softmax group
// each share every staged tile, so that keys and values enter an SM once for
// 256 rows.
//
// Warp roles (8 warps, 12 with NQ = 2):
//   warp 0     K producer, warp 6 V producer: a TMA box per (page, 64-column
//              chunk), a lane each, page ids read one tile ahead; they start
//              before the plan is known to be done
//   warps 1, 7 MMA issuers: S_j = Q K_j^T and O += P_j V_j, and the loads of Q
//              ahead of a piece's first scores.  Issuing a tile's
//              products, commits and waits takes one warp as long as a tile may
//              take, so two share it: NQ = 1 one the scores and one the values,
//              NQ = 2 a row tile each.  Warp 1 owns the tensor memory.
//   warps 2-5 (8-11) softmax, a TMEM lane quarter each: a thread per query row;
//              online base-2 softmax with a lazily moved maximum (O is rescaled
//              when it grows by more than 2^8); quarters without a used row skip
//              the arithmetic.  Warps 2-5 also zero the V rows that no query may
//              see (past the prefix end, unused nodes), so that what they hold
//              never meets a zero probability.
// Probabilities are rounded to bf16, the products' type, and summed unrounded in
// fp32: outputs are within 2.3e-3 relative (root mean square), 1.7e-3 of it their
// own rounding.
//
// The whole call: 64 requests x 16 nodes, prefixes of 512 to 8192, D = 256: 114 us,
// 5.2 TB/s, bound by the keys' and values' bytes.  96 requests x up to 61 nodes,
// prefixes of 251 to 2048, D = 128, 16 tokens a page: 85 us, 3.2 TB/s; a tile takes
// 0.9 us for its two row tiles, 0.67 us of it the MMAs, and the pieces' ends and
// joins 25 us of the call.  One token over 16384: 18 us, most of it the three
// launches' chain.
// Every wait is bounded; a timeout sets FLARE_DEV_WAIT_TIMEOUT, the CTA stops
// issuing work, writes nothing more, waits for its copies in flight, frees its
// tensor memory and exits.
#include <cudaTypedefs.h>

#include "common.cuh"
#include "kernels.h"
#include "pdl.cuh"
#include "tc.cuh"
#include "tree.cuh"
#include "tree_sched.cuh"

namespace flare {

namespace {

constexpr int kRowsT = 128;            // query rows of a row tile (TMEM lanes)
constexpr int kSmThreads = 128;        // softmax threads of a row tile
constexpr int kVWarpT = 6, kMma2WarpT = 7;
constexpr float kMoveMax = 8.0f;       // log2 units

template <int D, int NQ>
struct TreeCfg {
  static constexpr int kThreads = NQ == 1 ? 256 : 384;
  static constexpr int kChunks = D / 64;
  static constexpr int kTileBytes = kChunks * kTreeTile * 128;  // one K (or V) tile
  static constexpr int kQTile = kChunks * kRowsT * 128;         // one row tile's queries
  // K and V rings: what the queries leave of shared memory
  static constexpr int kKStages = D == 256 ? 2 : D == 128 ? (NQ == 2 ? 5 : 6) : 8;
  static constexpr int kVStages = D == 256 ? 3 : D == 128 ? (NQ == 2 ? 5 : 6) : 8;
  static constexpr int kSmem = NQ * kQTile + (kKStages + kVStages) * kTileBytes + 1024;
  // tensor memory columns, per row tile: O, then the S / P buffers
  static constexpr int kSBuf = D == 256 ? 4 : (NQ == 2 && D == 128 ? 2 : 3);
  static constexpr int kSCol = D;
  static constexpr int kRowCols = kSCol + kSBuf * kTreeTile;
  static constexpr int kTmemCols = NQ * kRowCols > 256 ? 512 : 256;
  static_assert(NQ * kRowCols <= 512, "tensor memory");
  static_assert(kSmem + 1024 <= 227 * 1024, "shared memory");
};

struct TreeShared {
  uint64_t k_full[8], k_empty[8], v_full[8], v_empty[8], v_fix[8];
  uint64_t s_full[2][4], p_full[2][4], pv_done[2][4];  // per row tile
  uint64_t q_full[2], o_final[2], o_free[2];
  uint64_t drain[2];  // after a timeout: every MMA issued has completed
  uint32_t tmem_base;
  int abort_flag;
  int last[2];  // whether this CTA's piece of an item ended last
};

__device__ __forceinline__ bool warp_wait_t(uint64_t* bar, uint32_t parity, const int* abort) {
  return __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, abort));
}

__device__ __forceinline__ bool aborted_t(const TreeShared& sh) {
  return *reinterpret_cast<const volatile int*>(&sh.abort_flag) != 0;
}

__device__ __forceinline__ void give_up(TreeShared& sh, int32_t* status) {
  if (!sh.abort_flag) {
    sh.abort_flag = 1;
    flag(status, FLARE_DEV_WAIT_TIMEOUT);
  }
}

// Barrier `id` over a row tile's 128 softmax threads, with an OR.
__device__ __forceinline__ bool group_or(uint32_t id, bool x) {
  int r;
  asm volatile(
      "{\n"
      " .reg .pred p, q;\n"
      " setp.ne.s32 p, %2, 0;\n"
      " bar.red.or.pred q, %1, 128, p;\n"
      " selp.s32 %0, 1, 0, q;\n"
      "}\n"
      : "=r"(r)
      : "r"(id), "r"((int)x)
      : "memory");
  return r != 0;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// 32 bytes, a memory sector, per thread and instruction: the output's rows are
// strided across a warp's lanes.
__device__ __forceinline__ void store32(void* p, const uint32_t (&x)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(x[0]),
               "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7])
               : "memory");
}

// A piece with what the roles ask of its request.
struct TreeItem {
  TreePiece w;
  int P, nodes, tiles;
  // tile j of the piece: whether it holds the tree's keys, and how many of its
  // rows are keys at all
  __device__ __forceinline__ bool is_tree(int j) const { return w.j0 + j == w.n - 1; }
  __device__ __forceinline__ int valid(int j) const {
    return is_tree(j) ? nodes : min(kTreeTile, P - (w.j0 + j) * kTreeTile);
  }
};

// The next piece of the span whose tree reaches node `node0`, a row tile's first.
__device__ __forceinline__ bool next_item(const TreeSoftmaxParams& p, TreeCursor& cur, int node0,
                                          TreeItem& it) {
  while (cur.next(p, it.w)) {
    it.nodes = p.node_len[it.w.r];
    if (node0 >= it.nodes) continue;
    it.P = p.prefix_len[it.w.r];
    it.tiles = it.w.j1 - it.w.j0;
    return true;
  }
  return false;
}

}  // namespace

template <int D, int NQ>
__global__ void __launch_bounds__(TreeCfg<D, NQ>::kThreads, 1)
    tree_softmax_tc_kernel(const __grid_constant__ TreeSoftmaxTc maps, TreeSoftmaxParams p) {
  using C = TreeCfg<D, NQ>;
  constexpr int kSB = C::kSBuf;
  extern __shared__ uint8_t smem_raw[];
  __shared__ TreeShared sh;
  uint8_t* Qs = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* Ks = Qs + NQ * C::kQTile;
  uint8_t* Vs = Ks + C::kKStages * C::kTileBytes;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int gang = blockIdx.x / p.row_tiles, mt = blockIdx.x % p.row_tiles;
  const int node0 = tree_rows(p, mt * NQ).node0;  // of the CTA's first row tile

  // the tensor maps, on their way while the span is worked out
  if (lane == 0) {
    if (warp == 0) tc::prefetch_tmap(&maps.kpool);
    if (warp == 1) tc::prefetch_tmap(&maps.q);
    if (warp == 2) tc::prefetch_tmap(&maps.kblk);
    if (warp == 3) tc::prefetch_tmap(&maps.vblk);
    if (warp == kVWarpT) tc::prefetch_tmap(&maps.vpool);
  }
  // barriers, a thread each: arrivals per phase
  {
    auto init = [&](int first, uint64_t* bars, int n, int count) {
      if (tid >= first && tid < first + n) tc::mbar_init(bars + tid - first, count);
    };
    init(0, sh.k_full, C::kKStages, 1);
    init(8, sh.k_empty, C::kKStages, NQ);  // a product per row tile
    init(16, sh.v_full, C::kVStages, 1);
    init(24, sh.v_empty, C::kVStages, NQ);
    init(32, sh.v_fix, C::kVStages, kSmThreads);
    init(40, &sh.s_full[0][0], 8, 1);
    init(48, &sh.p_full[0][0], 8, kSmThreads);
    init(56, &sh.pv_done[0][0], 8, 1);
    init(64, sh.q_full, 2, 1);
    init(66, sh.o_final, 2, 1);
    init(68, sh.o_free, 2, kSmThreads);
    init(70, sh.drain, 2, 1);
    if (tid == 72) sh.abort_flag = 0;
    if (tid < 96) tc::fence_mbar_init();
  }
  if (warp == 1) tc::tmem_alloc(&sh.tmem_base, C::kTmemCols);
  const TreeSpan span = tree_span(p, gang);
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = sh.tmem_base;
  TreeCursor cur = span.start;
  TreeItem it;

  if (warp == 0 || warp == kVWarpT) {
    // ------------------------------------------------------------ producers
    const int kv = warp == 0 ? 0 : 1;
    const CUtensorMap* pool_map = kv ? &maps.vpool : &maps.kpool;
    const CUtensorMap* blk_map = kv ? &maps.vblk : &maps.kblk;
    const int box_rows = p.page_size < kTreeTile ? p.page_size : kTreeTile;
    const int boxes = kTreeTile / box_rows;  // of a full tile
    const int ns = kv ? C::kVStages : C::kKStages;
    uint64_t* fulls = kv ? sh.v_full : sh.k_full;
    uint64_t* empties = kv ? sh.v_empty : sh.k_empty;
    uint8_t* ring = kv ? Vs : Ks;
    const int bx = lane / C::kChunks, ch = lane % C::kChunks;  // this lane's box of a tile
    bool ok = true;
    int g = 0;  // running tile count
    while (ok && next_item(p, cur, node0, it)) {
      const int32_t* table = p.page_table + (size_t)it.w.r * p.max_pages;
      // the page of this lane's box in tile j (0 where the tile has no such box)
      auto page_of = [&](int j) -> int {
        const int tok = (it.w.j0 + j) * kTreeTile + bx * box_rows;
        return j < it.tiles && bx < boxes && !it.is_tree(j) && tok < it.P ? table[tok / p.page_size]
                                                                         : 0;
      };
      int page = page_of(0);
      for (int j = 0; j < it.tiles; ++j, ++g) {
        const int page_next = page_of(j + 1);
        const int st = g % ns;
        const uint32_t ph = (uint32_t)(g / ns) & 1u;
        uint8_t* dst = ring + st * C::kTileBytes;
        if (!warp_wait_t(&empties[st], ph ^ 1u, &sh.abort_flag)) {
          ok = false;
          break;
        }
        if (it.is_tree(j)) {
          if (lane == 0) {
            tc::mbar_expect_tx(&fulls[st], C::kTileBytes);
#pragma unroll
            for (int c = 0; c < C::kChunks; ++c)
              tc::tma_load_4d(dst + c * (kTreeTile * 128), blk_map, &fulls[st], c * 64, it.w.kvh,
                              0, it.w.r);
          }
        } else {
          const int tok0 = (it.w.j0 + j) * kTreeTile;
          const int nbox = (min(kTreeTile, it.P - tok0) + box_rows - 1) / box_rows;
          if (lane == 0)
            tc::mbar_expect_tx(&fulls[st], (uint32_t)(C::kChunks * nbox * box_rows * 128));
          __syncwarp();
          if (bx < nbox)
            tc::tma_load_4d(dst + ch * (kTreeTile * 128) + bx * box_rows * 128, pool_map,
                            &fulls[st], ch * 64, (tok0 + bx * box_rows) % p.page_size, it.w.kvh,
                            page);
        }
        page = page_next;
      }
    }
    if (!ok && lane == 0) give_up(sh, p.dev_status);
    // on the way out every copy issued has landed (a consumer that gave up may
    // have left some in flight)
    if (aborted_t(sh)) {
      for (int s = 0; s < ns && s < g; ++s) {
        const int last = g - 1 - ((g - 1 - s) % ns + ns) % ns;  // last tile issued into slot s
        if (last >= 0) tc::mbar_wait(&fulls[s], (uint32_t)(last / ns) & 1u, nullptr, 100000000ull);
      }
    }
  } else if (warp == 1 || warp == kMma2WarpT) {
    // ------------------------------------------------------------ MMA issuers
    // The whole warp walks the loop with the same values and one elected thread
    // issues, so that descriptors stay in uniform registers: issued from a
    // branch on one lane, each MMA costs some 60 cycles of moves into them.
    const int t = NQ == 2 && warp != 1 ? 1 : 0;  // of row tile t
    const bool scores = NQ == 2 || warp == 1, values = NQ == 2 || warp != 1;
    const TreeRows rows = tree_rows(p, mt * NQ + t);
    const int box_heads = min(p.G, kRowsT);
    const uint32_t q_bytes = (uint32_t)(C::kChunks * 128 * box_heads * rows.nodes);
    const uint32_t base = tmem + t * C::kRowCols;
    const uint32_t id_s = tc::idesc_bf16(kRowsT, kTreeTile, false, false);
    const uint32_t id_o = tc::idesc_bf16(kRowsT, D, false, true);
    const uint64_t kdesc0 = tc::sdesc_sw128(tc::smem_u32(Ks), 16, 1024);
    const uint64_t vdesc0 = tc::sdesc_sw128(tc::smem_u32(Vs), kTreeTile * 128, 1024);
    const uint64_t qdesc0 = tc::sdesc_sw128(tc::smem_u32(Qs + t * C::kQTile), 16, 1024);
    bool ok = true;
    int g = 0;              // running tile count of the rings
    int gt = 0, kt = 0;     // of this row tile's buffers, and its pieces
    uint32_t fix_par = 0u;  // per V slot: parity of its next zeroed tile
    bool q_out = false;     // queries in flight
    while (ok && next_item(p, cur, node0, it)) {
      const int n = it.tiles;
      auto k_tile = [&](int j) {
        return warp_wait_t(&sh.k_full[(g + j) % C::kKStages],
                           (uint32_t)((g + j) / C::kKStages) & 1u, &sh.abort_flag);
      };
      auto v_tile = [&](int j) {
        const int st = (g + j) % C::kVStages;
        if (!warp_wait_t(&sh.v_full[st], (uint32_t)((g + j) / C::kVStages) & 1u, &sh.abort_flag))
          return false;
        if (it.valid(j) < kTreeTile) {
          if (!warp_wait_t(&sh.v_fix[st], (fix_par >> st) & 1u, &sh.abort_flag)) return false;
          fix_par ^= 1u << st;
        }
        return true;
      };
      if (rows.node0 >= it.nodes) {  // no rows of this item: pass its tiles on
        for (int j = 0; j < n && ok; ++j) {
          ok = k_tile(j) && v_tile(j);
          if (ok && lane == 0) {
            tc::mbar_arrive(&sh.k_empty[(g + j) % C::kKStages]);
            tc::mbar_arrive(&sh.v_empty[(g + j) % C::kVStages]);
          }
          __syncwarp();
        }
        g += n;
        continue;
      }
      if (scores) {
        // the queries, once the last piece's scores have read theirs
        if (kt > 0)
          ok = warp_wait_t(&sh.s_full[t][(gt - 1) % kSB], (uint32_t)((gt - 1) / kSB) & 1u,
                           &sh.abort_flag);
        if (!ok) break;
        if (tc::elect_one()) {
          uint8_t* dst = Qs + t * C::kQTile;
          tc::mbar_expect_tx(&sh.q_full[t], q_bytes);
#pragma unroll
          for (int c = 0; c < C::kChunks; ++c)
            tc::tma_load_4d(dst + c * (kRowsT * 128), &maps.q, &sh.q_full[t], c * 64,
                            it.w.kvh * p.G + rows.head0, rows.node0, it.w.r);
        }
        __syncwarp();
        q_out = true;
        ok = warp_wait_t(&sh.q_full[t], (uint32_t)kt & 1u, &sh.abort_flag);
        if (!ok) break;
        q_out = false;
      }
      auto issue_s = [&](int j) -> bool {  // S_j = Q K_j^T
        if (!k_tile(j)) return false;
        tc::fence_after_sync();
        const int st = (g + j) % C::kKStages, sb = (gt + j) % kSB;
        const uint64_t kd = kdesc0 + (uint64_t)((st * C::kTileBytes) >> 4);
        if (tc::elect_one()) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint64_t kdk =
                kd + (uint64_t)(((kk >> 2) * (kTreeTile * 128) + (kk & 3) * 32) >> 4);
            tc::mma_bf16_ss(base + C::kSCol + sb * kTreeTile,
                            qdesc0 + (uint64_t)(((kk >> 2) * (kRowsT * 128) + (kk & 3) * 32) >> 4),
                            kdk, id_s, kk > 0 ? 1u : 0u);
          }
          tc::mma_commit(&sh.s_full[t][sb]);
          tc::mma_commit(&sh.k_empty[st]);
        }
        __syncwarp();
        return true;
      };
      auto issue_pv = [&](int j) -> bool {  // O += P_j V_j
        const int st = (g + j) % C::kVStages, pb = (gt + j) % kSB;
        if (!warp_wait_t(&sh.p_full[t][pb], (uint32_t)((gt + j) / kSB) & 1u, &sh.abort_flag))
          return false;
        // the first product of a piece overwrites O: the previous one's must be out
        if (j == 0 && kt > 0 &&
            !warp_wait_t(&sh.o_free[t], (uint32_t)(kt - 1) & 1u, &sh.abort_flag))
          return false;
        if (!v_tile(j)) return false;
        tc::fence_after_sync();
        const uint64_t vd = vdesc0 + (uint64_t)((st * C::kTileBytes) >> 4);
        if (tc::elect_one()) {
#pragma unroll
          for (int kk = 0; kk < kTreeTile / 16; ++kk)
            tc::mma_bf16_ts(base, base + C::kSCol + pb * kTreeTile + kk * 8,
                            vd + (uint64_t)(kk * (2048 >> 4)), id_o, (j > 0 || kk > 0) ? 1u : 0u);
          tc::mma_commit(&sh.pv_done[t][pb]);
          tc::mma_commit(&sh.v_empty[st]);
        }
        __syncwarp();
        return true;
      };
      if constexpr (NQ == 2) {
        // MMAs of one thread execute in issue order, so an S buffer can be
        // rewritten once the product that reads its probabilities was issued:
        // kSB scores ahead, then P V_j and S_j+kSB in turn.  No wait stands behind
        // this, for products of two shapes; the calls' repetitions bit for bit do.
        for (int j = 0; j < kSB && j < n && ok; ++j) ok = issue_s(j);
        for (int j = 0; j < n && ok; ++j) {
          ok = issue_pv(j);
          if (ok && j + kSB < n) ok = issue_s(j + kSB);
        }
      } else if (scores) {
        for (int j = 0; j < n && ok; ++j) {
          const int gg = gt + j;  // the buffer's last probabilities have been read
          if (gg >= kSB)
            ok = warp_wait_t(&sh.pv_done[t][gg % kSB], (uint32_t)(gg / kSB - 1) & 1u,
                             &sh.abort_flag);
          ok = ok && issue_s(j);
        }
      } else {
        for (int j = 0; j < n && ok; ++j) ok = issue_pv(j);
      }
      if (!ok) break;
      if (values && tc::elect_one()) tc::mma_commit(&sh.o_final[t]);
      __syncwarp();
      gt += n;
      ++kt;
      g += n;
    }
    if (!ok && lane == 0) give_up(sh, p.dev_status);
    __syncwarp();
    if (aborted_t(sh)) {
      if (q_out) tc::mbar_wait(&sh.q_full[t], (uint32_t)kt & 1u, nullptr, 100000000ull);
      uint64_t* drain = &sh.drain[warp == 1 ? 0 : 1];
      if (tc::elect_one()) {
        tc::mma_commit(drain);
        tc::mbar_wait(drain, 0u, nullptr, 100000000ull);
      }
      __syncwarp();
    }
  } else {
    // ------------------------------------------------------------ softmax warps
    const int quarter = warp & 3, t = NQ == 2 && warp >= 8 ? 1 : 0;  // of row tile t
    const int row = quarter * 32 + lane;
    const TreeRows rows = tree_rows(p, mt * NQ + t);
    const int node = rows.node(row), head = rows.head(row);
    const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
    const uint32_t tmem_o = tmem + t * C::kRowCols, tmem_s = tmem_o + C::kSCol;
    const bool out32 = ((uintptr_t)p.out & 31u) == 0;  // the caller's tensors: 16 bytes at least

    bool ok = true;
    int g = 0;  // running tile count (of row tile 0: the rings' too)
    // V rows of tile j that no query may see.  The slot cannot be refilled before
    // this tile's product, which waits for these threads, so the parity wait is
    // exact, though not every tile is waited for, once the slot's last tile has been
    // read: with more score buffers than V slots these threads may be ahead of that.
    auto zero_v = [&](int j) -> bool {
      const int valid = it.valid(j);
      if (t != 0 || valid == kTreeTile) return true;
      const int gg = g + j, st = gg % C::kVStages;
      if constexpr (kSB > C::kVStages) {
        const int last = gg - C::kVStages;
        if (last >= 0 && !warp_wait_t(&sh.pv_done[t][last % kSB], (uint32_t)(last / kSB) & 1u,
                                      &sh.abort_flag))
          return false;
      }
      if (!warp_wait_t(&sh.v_full[st], (uint32_t)(gg / C::kVStages) & 1u, &sh.abort_flag))
        return false;
      uint8_t* dst = Vs + st * C::kTileBytes;
      const int n16 = (kTreeTile - valid) * 8;  // 16-byte pieces per chunk
      for (int c = 0; c < C::kChunks; ++c)
        for (int e = row; e < n16; e += kSmThreads)
          *reinterpret_cast<uint4*>(dst + c * (kTreeTile * 128) + (valid + e / 8) * 128 +
                                    (e % 8) * 16) = make_uint4(0u, 0u, 0u, 0u);
      tc::fence_async_smem();
      tc::mbar_arrive(&sh.v_fix[st]);
      return true;
    };
    bool have = next_item(p, cur, rows.node0, it);
    pdl_wait();  // the plan: paths, and which requests are bad
    if (tid == 64) pdl_launch_next();
    auto path_of = [&](const TreeItem& x) {
      return rows.used(row, x.nodes) ? p.anc[(size_t)x.w.r * p.N + node] : 0ull;
    };
    uint64_t path = have ? path_of(it) : 0ull;
    int bad = have ? p.bad[it.w.r] : 0;
    for (int k = 0; have; ++k) {
      const bool live = rows.used(row, it.nodes);
      const bool warp_live = __any_sync(0xffffffffu, live);
      float m_run = -INFINITY, l_run = 0.f;
      for (int j = 0; j < it.tiles; ++j) {
        const int gg = g + j, sb = gg % kSB;
        if (!warp_wait_t(&sh.s_full[t][sb], (uint32_t)(gg / kSB) & 1u, &sh.abort_flag)) {
          ok = false;
          break;
        }
        if (!warp_live) {  // nobody reads these rows' output
          ok = zero_v(j);
          if (!ok) break;
          tc::mbar_arrive(&sh.p_full[t][sb]);
          continue;
        }
        tc::fence_after_sync();
        const uint32_t sbuf = tmem_s + lane_off + sb * kTreeTile;
        uint32_t sr[kTreeTile];
#pragma unroll
        for (int c = 0; c < kTreeTile; c += 16)
          tc::tmem_ld16(sbuf + c, *reinterpret_cast<uint32_t(*)[16]>(&sr[c]));
        tc::tmem_ld_wait();
        const int valid = it.valid(j);
        if (it.is_tree(j)) {
#pragma unroll
          for (int c = 0; c < kTreeTile; ++c)
            if (!((path >> c) & 1)) sr[c] = 0xff800000u;  // -inf
        } else if (valid < kTreeTile) {
#pragma unroll
          for (int c = 0; c < kTreeTile; ++c)
            if (c >= valid) sr[c] = 0xff800000u;
        }
        // tile maximum of the raw scores (scale > 0 keeps the order, and -inf)
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < kTreeTile; c += 2)
          mx[c / 2 & 3] = max3(mx[c / 2 & 3], __uint_as_float(sr[c]), __uint_as_float(sr[c + 1]));
        const float mt_ = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        const float m_new = fmaxf(m_run, mt_ * p.scale_log2);
        // (rows in use decide: what the others hold is not defined)
        const bool need = j == 0 || (live && m_new > m_run + kMoveMax);
        const bool move = __any_sync(0xffffffffu, need);
        const float m_use = move ? m_new : m_run;
        const float corr = j == 0 ? 0.f : tc::ex2(m_run - m_use);
        // a row that sees nothing of its tiles so far: every probability 0
        const float neg_m = m_use == -INFINITY ? 0.f : -m_use;
        const uint64_t scale2 = f2_dup(p.scale_log2), neg2 = f2_dup(neg_m);
        uint64_t sum = 0ull;
        uint32_t pk[kTreeTile / 2];
#pragma unroll
        for (int c = 0; c < kTreeTile; c += 2) {
          float p0, p1;
          f2_split(f2_fma(f2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1])), scale2, neg2), p0,
                   p1);
          p0 = tc::ex2(p0);
          p1 = tc::ex2(p1);
          sum = f2_add(sum, f2(p0, p1));
          const __nv_bfloat162 h2 = __floats2bfloat162_rn(p0, p1);
          pk[c / 2] = *reinterpret_cast<const uint32_t*>(&h2);
        }
        float sum0, sum1;
        f2_split(sum, sum0, sum1);
        l_run = j == 0 ? sum0 + sum1 : l_run * corr + (sum0 + sum1);
        if (move && j >= 1) {  // rescale O, the previous tile's product done
          const int pb = (gg - 1) % kSB;
          if (!warp_wait_t(&sh.pv_done[t][pb], (uint32_t)((gg - 1) / kSB) & 1u, &sh.abort_flag)) {
            ok = false;
            break;
          }
          tc::fence_after_sync();
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            uint32_t o[16];
            tc::tmem_ld16(tmem_o + lane_off + c, o);
            tc::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * corr);
            tc::tmem_st16(tmem_o + lane_off + c, o);
          }
        }
        m_run = m_use;
#pragma unroll
        for (int c = 0; c < kTreeTile / 2; c += 16)
          tc::tmem_st16(sbuf + c, *reinterpret_cast<uint32_t(*)[16]>(&pk[c]));
        tc::tmem_st_wait();
        ok = zero_v(j);
        if (!ok) break;
        tc::fence_before_sync();
        tc::mbar_arrive(&sh.p_full[t][sb]);
      }
      g += it.tiles;
      // what the next piece needs first, in flight while this one's output leaves
      TreeItem nx;
      const bool more = next_item(p, cur, rows.node0, nx), skip = bad != 0;
      if (more) {
        path = path_of(nx);
        bad = p.bad[nx.w.r];
      }
      if (tid == 64 && mt == 0 && !skip) tree_list_cut(p, span, it.w);
      if (ok && aborted_t(sh)) ok = false;
      if (ok && !warp_wait_t(&sh.o_final[t], (uint32_t)k & 1u, &sh.abort_flag)) ok = false;
      if (group_or(2 + t, !ok)) {  // the row tile's four warps agree
        ok = false;
        break;
      }
      tc::fence_after_sync();
      const bool whole = it.w.whole();
      const float inv = l_run > 0.f ? 1.f / l_run : 0.f;
      const float l2 = l_run > 0.f ? m_run + log2f(l_run) : -INFINITY;
      // the gangs that share the item
      int g0 = gang, g1 = gang;
      if (!whole) tree_sharers(span, it.w, g0, g1);
      const bool joins = !whole && !skip && g1 - g0 < kTreeJoin;
      bool store = !whole && !skip, merge = false;  // a partial output; the item's
      int32_t* count = p.counts + ((size_t)g0 * p.row_tiles + mt) * NQ + t;
      if (joins) {  // with every other piece stored, this one need not be
        if (row == 0)
          sh.last[t] = atomicAdd(count, 0) == g1 - g0;
        tc::named_bar_sync(2 + t, kSmThreads);
        merge = sh.last[t] != 0;
        store = !merge;
      }
      if (store && warp_live) {
        const size_t part = tree_part(p, gang, g0, mt);
        const int trow = t * kRowsT + row;
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 64) {
          uint32_t o[64];
#pragma unroll
          for (int c = 0; c < 64; c += 16)
            tc::tmem_ld16(tmem_o + lane_off + c0 + c, *reinterpret_cast<uint32_t(*)[16]>(&o[c]));
          tc::tmem_ld_wait();
          if (!live) continue;
#pragma unroll
          for (int c = 0; c < 64; c += 4)
            *tree_part_at(p, part, trow, (c0 + c) / 4) = make_float4(
                __uint_as_float(o[c]) * inv, __uint_as_float(o[c + 1]) * inv,
                __uint_as_float(o[c + 2]) * inv, __uint_as_float(o[c + 3]) * inv);
        }
        if (live) p.part_lse[part + trow] = l2;
      }
      if (joins && store) {
        __threadfence();
        tc::named_bar_sync(2 + t, kSmThreads);
        if (row == 0) sh.last[t] = atomicAdd(count, 1) == g1 - g0;
        tc::named_bar_sync(2 + t, kSmThreads);
        merge = sh.last[t] != 0;
      }
      if ((whole && !skip) || merge) {
        if (warp_live) {
          if (merge) __threadfence();
          // weights of the item's pieces, in gang order
          float wt[kTreeJoin];
          float top = -INFINITY, den = 0.f;
          const int trow = t * kRowsT + row;
#pragma unroll
          for (int u = 0; u < kTreeJoin; ++u) {
            wt[u] = -INFINITY;
            if (g0 + u <= g1 && live)
              wt[u] = g0 + u == gang ? l2 : __ldcg(p.part_lse + tree_part(p, g0 + u, g0, mt) + trow);
            top = fmaxf(top, wt[u]);
          }
#pragma unroll
          for (int u = 0; u < kTreeJoin; ++u) {
            wt[u] = wt[u] == -INFINITY ? 0.f : exp2f(wt[u] - top);
            den += wt[u];
          }
          const float norm = den > 0.f ? 1.f / den : 0.f;
          auto weight = [&](int u) {
            return (u == 0 ? wt[0] : u == 1 ? wt[1] : u == 2 ? wt[2] : wt[3]) * norm;
          };
          const size_t orow = ((size_t)it.w.r * p.N + node) * p.Hq + it.w.kvh * p.G + head;
          __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + orow * D;
          auto put = [&](int c, const float* x) {  // columns c .. c + 15 of the output
            uint32_t h[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const __nv_bfloat162 h2 = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
              h[i] = *reinterpret_cast<const uint32_t*>(&h2);
            }
            if (out32) {
              store32(out + c, h);
            } else {
              *reinterpret_cast<uint4*>(out + c) = make_uint4(h[0], h[1], h[2], h[3]);
              *reinterpret_cast<uint4*>(out + c + 8) = make_uint4(h[4], h[5], h[6], h[7]);
            }
          };
          constexpr int kCols = NQ == 1 ? 64 : 32;  // at a time: as registers allow
          // the other pieces' columns, kCols at a time: every load of a batch in
          // flight before the first is used
#pragma unroll 1
          for (int c0 = 0; c0 < D; c0 += kCols) {
            uint32_t o[kCols];
#pragma unroll
            for (int c = 0; c < kCols; c += 16)
              tc::tmem_ld16(tmem_o + lane_off + c0 + c, *reinterpret_cast<uint32_t(*)[16]>(&o[c]));
            tc::tmem_ld_wait();
            float acc[kCols];
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[c] = __uint_as_float(o[c]) * inv;
            if (!whole) {
              const float own = weight(gang - g0);
              if (gang == g0) {
#pragma unroll
                for (int c = 0; c < kCols; ++c) acc[c] *= own;
              } else {  // its turn comes later: back to tensor memory meanwhile
#pragma unroll
                for (int c = 0; c < kCols; ++c) acc[c] = 0.f;
              }
#pragma unroll 1
              for (int u = gang == g0 ? 1 : 0; u <= g1 - g0; ++u) {
                const float f = weight(u);
                if (g0 + u == gang) {
#pragma unroll
                  for (int c = 0; c < kCols; c += 16)
                    tc::tmem_ld16(tmem_o + lane_off + c0 + c,
                                  *reinterpret_cast<uint32_t(*)[16]>(&o[c]));
                  tc::tmem_ld_wait();
#pragma unroll
                  for (int c = 0; c < kCols; ++c)
                    acc[c] = fmaf(f, __uint_as_float(o[c]) * inv, acc[c]);
                } else if (live && f > 0.f) {
                  const float4* src =
                      tree_part_at(p, tree_part(p, g0 + u, g0, mt), trow, c0 / 4);
                  float4 x[kCols / 4];
#pragma unroll
                  for (int c = 0; c < kCols / 4; ++c) x[c] = __ldcg(src + (size_t)c * p.tile_rows);
#pragma unroll
                  for (int c = 0; c < kCols / 4; ++c) {
                    acc[4 * c] = fmaf(f, x[c].x, acc[4 * c]);
                    acc[4 * c + 1] = fmaf(f, x[c].y, acc[4 * c + 1]);
                    acc[4 * c + 2] = fmaf(f, x[c].z, acc[4 * c + 2]);
                    acc[4 * c + 3] = fmaf(f, x[c].w, acc[4 * c + 3]);
                  }
                }
              }
            }
            if (!live) continue;
#pragma unroll
            for (int c = 0; c < kCols; c += 16) put(c0 + c, acc + c);
          }
          if (live && p.lse)
            p.lse[orow] = (whole ? l2 : den > 0.f ? top + log2f(den) : -INFINITY) * 0.6931471805599453f;
        }
      }
      tc::fence_before_sync();
      tc::mbar_arrive(&sh.o_free[t]);
      it = nx;
      have = more;
    }
    if (!ok) give_up(sh, p.dev_status);
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, C::kTmemCols);
  }
  pdl_wait();  // also where the span was empty
}

// ------------------------------------------------------------------ host side

namespace {

PFN_cuTensorMapEncodeTiled_v12000 tree_encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault,
                                         &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  }();
  return fn;
}

bool encode(CUtensorMap* m, const void* ptr, const cuuint64_t (&dims)[4],
            const cuuint64_t (&strides)[3], const cuuint32_t (&box)[4]) {
  auto fn = tree_encode_fn();
  if (!fn) return false;
  const cuuint32_t es[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) ==
         CUDA_SUCCESS;
}

template <int D, int NQ>
cudaError_t launch_tc_d(const TreeSoftmaxParams& p, const TreeSoftmaxTc& maps,
                        cudaStream_t stream) {
  using C = TreeCfg<D, NQ>;
  cudaError_t e = cudaFuncSetAttribute(tree_softmax_tc_kernel<D, NQ>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
  if (e != cudaSuccess) return e;
  e = pdl_launch(tree_softmax_tc_kernel<D, NQ>, dim3((unsigned)(p.gangs * p.row_tiles)),
                 C::kThreads, C::kSmem, stream, true, 1, maps, p);
  note_launches(1);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t prepare_tree_softmax_tc(const TreeSoftmaxParams& p, TreeSoftmaxTc* m) {
  const cuuint64_t D = p.D, row = D * 2;
  {  // (D, heads, N, R): the nodes' rows; a box is 64 columns of a row tile
    const cuuint64_t dims[4] = {D, (cuuint64_t)p.Hq, (cuuint64_t)p.N, (cuuint64_t)p.R};
    const cuuint64_t str[3] = {row, p.Hq * row, (cuuint64_t)p.N * p.Hq * row};
    const cuuint32_t heads = p.G < kRowsT ? p.G : kRowsT;
    const cuuint32_t box[4] = {64, heads, p.G < kRowsT ? kRowsT / heads : 1, 1};
    if (!encode(&m->q, p.q, dims, str, box)) return cudaErrorInvalidValue;
  }
  {
    const cuuint64_t dims[4] = {D, (cuuint64_t)p.Hkv, (cuuint64_t)p.N, (cuuint64_t)p.R};
    const cuuint64_t str[3] = {row, p.Hkv * row, (cuuint64_t)p.N * p.Hkv * row};
    const cuuint32_t box[4] = {64, 1, kTreeTile, 1};
    if (!encode(&m->kblk, p.k_blk, dims, str, box) || !encode(&m->vblk, p.v_blk, dims, str, box))
      return cudaErrorInvalidValue;
  }
  // (D, page rows, kv heads, pages).  Page ids are checked beside the stream: one
  // outside the pool reads as zeros.  Without a pool the maps show one row of the
  // nodes' tensors.
  const bool none = p.num_pages == 0 || p.max_pages == 0;
  const cuuint64_t dims[4] = {D, (cuuint64_t)(none ? 1 : p.page_size),
                              (cuuint64_t)(none ? 1 : p.Hkv), (cuuint64_t)(none ? 1 : p.num_pages)};
  const cuuint64_t str[3] = {row, p.page_size * row, (cuuint64_t)p.Hkv * p.page_size * row};
  const cuuint32_t box[4] = {64, (cuuint32_t)(p.page_size < kTreeTile ? p.page_size : kTreeTile), 1,
                             1};
  if (!encode(&m->kpool, none ? p.k_blk : p.k_pool, dims, str, box) ||
      !encode(&m->vpool, none ? p.v_blk : p.v_pool, dims, str, box))
    return cudaErrorInvalidValue;
  return cudaSuccess;
}

cudaError_t launch_tree_softmax_tc(const TreeSoftmaxParams& p, const TreeSoftmaxTc& maps,
                                   cudaStream_t stream) {
  const bool two = p.tile_rows == 2 * kRowsT;
  switch (p.D) {
    case 64: return two ? launch_tc_d<64, 2>(p, maps, stream) : launch_tc_d<64, 1>(p, maps, stream);
    case 128:
      return two ? launch_tc_d<128, 2>(p, maps, stream) : launch_tc_d<128, 1>(p, maps, stream);
    case 256: return launch_tc_d<256, 1>(p, maps, stream);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace flare
