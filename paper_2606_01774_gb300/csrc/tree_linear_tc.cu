// Gated delta rule along the paths of a drafted tree on tcgen05 tensor cores:
// bf16 activations, 128 x 128 states, persistent CTAs.
//
// tree_linear.cu has the system that a tree's paths unroll to.  For one
// (request, value head) item, with BM = 16, 32 or 64 rows for the tree's nodes:
//   MMA  W^T = S0^T [K; Q]^T   M = 128 (value columns on lanes), N = 2 BM, K = 128
//        G   = [K; Q] K^T      M = 128 (rows on lanes), N = BM, over S0^T
//   A[i][j] = beta_i exp(gamma_i - gamma_j) G[i][j]     for j on i's path, j != i
//   M[i][j] = exp(gamma_i - gamma_j) G[BM + i][j]       for j on i's path
//   X_i = beta_i (v_i - exp(gamma_i) W^T[.][i]),  Y_i = exp(gamma_i) W^T[.][BM + i]
//   for i = 0, 1, ...   (thread c owns value column c; parents come first)
//     delta_i = X_i - sum_j A[i][j] delta_j,   out_i = scale (Y_i + sum_j M[i][j] delta_j)
// The nodes go in blocks of 16.  Inside a block substitution and readout run on
// the CUDA cores in one pass, with A and M side by side as pairs (-A, M), so
// that one packed multiply-add carries a delta into both sums.  From a finished
// block to the later ones,
//   MMA  [X | Y]^T (later) += delta^T [-A | M]^T        M = 128, N = 16 .. 48, K = 16
// with deltas and tables as bf16 high and low parts, three products each: both
// sums gather in tensor memory where the first MMA left X and Y.  (All on the
// CUDA cores, 61 nodes were bound by reading the tables from shared memory,
// 26 us a call of 192 items against 13.5, the state then rounded once.)
// The state, too, enters W as bf16 high and low parts (to about 2^-16, two products
// a step): rounded once, outputs were off by 2.6e-3 relative where their own
// rounding to bf16 makes 1.7e-3.
//
// Bound by the state's bytes: 64 KiB an item, so a CTA's life is organised
// around its copies.  Warp 4 runs ahead: it finds the next item, streams its
// state in 16 KiB pieces through a ring, its keys, queries and values by TMA,
// works out its paths and gates (pointer doubling), and issues the MMAs as the
// pieces become operands.  Warps 0-3 turn pieces into the bf16 operand S0^T in
// tensor memory, then tables, substitution and readout.  BM <= 32: 128
// tensor-memory columns, four (BM = 16) or three CTAs per SM; BM = 64: two.
// 64 requests x 16 nodes x 32 heads: 32.2 us, 4.9 TB/s; 6 x 61 nodes: 13.3 us.
// Every wait is bounded; on a timeout the CTA sets FLARE_DEV_WAIT_TIMEOUT,
// lets its copies and MMAs land, frees its tensor memory and exits.
#include <cudaTypedefs.h>

#include "common.cuh"
#include "kernels.h"
#include "tc.cuh"
#include "tree.cuh"

namespace flare {

namespace {

constexpr int kTlD = 128;          // d_k = d_v
constexpr int kTlCompute = 128;    // warps 0-3: a thread per value column
constexpr int kTlThreads = 160;    // and the producer warp
constexpr int kPieceRows = 32;     // state rows per ring piece
constexpr int kPieceBytes = kPieceRows * kTlD * 4;
constexpr int kPieces = kTlD / kPieceRows;  // per item

// What the producer warp works out for an item.  Three buffers: the item at
// work, the next one, whose state is on its way, and the one after, worked out
// while the first is in its readout.
template <int BM>
struct TlMeta {
  alignas(16) float gam2[BM];  // gamma_i log2(e)
  float beta[BM];
  uint64_t anc[BM];
  int item, n;                 // item < 0: no more; n < 0: skipped (a bad tree)
};

template <int BM>
struct TlCfg {
  // CTAs per SM, and state pieces in flight in each.  BM = 16: more CTAs overlap
  // more compute phases than deeper rings do (64 requests of 16 nodes: 3 CTAs with 4
  // pieces 34.0 us, 4 with 2 33.1 us)
  static constexpr int kCtas = BM == 64 ? 2 : BM == 32 ? 3 : 4;
  static constexpr int kBlocks = BM / 16;
  static constexpr int kRing = BM == 64 ? 3 : 2;
  static constexpr int kKQ = 2 * 2 * BM * 128;                 // 2 chunks of [K; Q] rows x 128 B
  // 2 chunks of value rows x 128 B; BM = 16: in registers
  static constexpr int kV = BM == 16 ? 0 : 2 * BM * 128;
  static constexpr int kDiag = kBlocks * 16 * 16 * 8;          // pairs (-A, M) inside blocks
  // -A high, low, M high, low between blocks: rows 16 .. BM - 1, K-major SW128
  static constexpr int kCross = (BM - 16) * 128;
  // BM = 64: the tables take the key / query buffer's place
  static constexpr bool kOverlay = BM == 64;
  static constexpr int kTables = kDiag + 4 * kCross;
  static constexpr int oKQ = 0;
  static constexpr int oRing = kKQ;
  static constexpr int oCross = kOverlay ? 0 : oRing + kRing * kPieceBytes;
  static constexpr int oDiag = oCross + 4 * kCross;
  static constexpr int oV = kOverlay ? oRing + kRing * kPieceBytes : oDiag + kDiag;
  static constexpr int oShared = oV + kV;
  static_assert(!kOverlay || kTables <= kKQ, "tables over keys and queries");
  static constexpr int kTmem = BM == 64 ? 256 : 128;
  // state pieces that tensor memory holds as operands beside W^T, 32 columns each
  static constexpr int kOps = (kTmem - 2 * BM) / 32 < kPieces ? (kTmem - 2 * BM) / 32 : kPieces;
};

template <int BM>
struct alignas(16) TlShared {
  TlMeta<BM> meta[3];
  uint64_t full[4], empty[4];  // ring pieces
  uint64_t kq_full, v_full, done, mma_done, upd, meta_full[3];  // done: an item's readout
  uint64_t op_free[2];  // the products with the first pieces, whose columns later ones take
  uint32_t tmem_base;
  int abort_flag;
};

template <int BM>
constexpr int tl_smem() {
  return TlCfg<BM>::oShared + (int)sizeof(TlShared<BM>);
}

struct TlMaps {
  CUtensorMap k, q;  // (128, Hk, N, R) box (64, 1, BM, 1), 128-byte swizzle
  CUtensorMap v;     // (128, Hv, N, R) box (64, 1, BM, 1), no swizzle
};

// Word offset of the pairs of columns 2 u, 2 u + 1 of row `row` of a block's 16 x
// 16 pairs, whose 16-byte units are XOR-swizzled by the row (a warp writes a row
// per lane).
__device__ __forceinline__ int tl_at(int row, int u) {
  return row * 32 + ((u ^ (row & 7)) << 2);
}

// x = hi + lo to about 2^-16 relative, each a bf16 pair (a low, b high).  The high
// parts are cut off, not rounded: one conversion less.
__device__ __forceinline__ void tl_split(float a, float b, uint32_t& hi, uint32_t& lo) {
  const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
  hi = __byte_perm(x, y, 0x7632);
  const __nv_bfloat162 l = __floats2bfloat162_rn(a - __uint_as_float(x & 0xffff0000u),
                                                 b - __uint_as_float(y & 0xffff0000u));
  lo = *reinterpret_cast<const uint32_t*>(&l);
}

__device__ __forceinline__ bool tl_warp_wait(uint64_t* bar, uint32_t parity, const int* abort) {
  return __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, abort));
}

// OR of a predicate over the 128 compute threads, with barrier semantics.
__device__ __forceinline__ bool tl_compute_or(bool x) {
  int r;
  asm volatile(
      "{\n"
      " .reg .pred p, q;\n"
      " setp.ne.s32 p, %1, 0;\n"
      " bar.red.or.pred q, 1, 128, p;\n"
      " selp.s32 %0, 1, 0, q;\n"
      "}\n"
      : "=r"(r)
      : "r"((int)x)
      : "memory");
  return r != 0;
}

__device__ __forceinline__ uint32_t tl_pack(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace

template <int BM>
__global__ void __launch_bounds__(kTlThreads, TlCfg<BM>::kCtas)
    tree_linear_tc_kernel(const __grid_constant__ TlMaps maps, GdrParams p) {
  using C = TlCfg<BM>;
  // no static shared memory: the dynamic window starts 1024-byte aligned, as
  // the swizzled operands need (checked below)
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  TlShared<BM>& sh = *reinterpret_cast<TlShared<BM>*>(smem_raw + C::oShared);
  uint8_t* KQ = smem_raw + C::oKQ;
  uint8_t* ring = smem_raw + C::oRing;
  float* Tp = reinterpret_cast<float*>(smem_raw + C::oDiag);
  uint8_t* Cross = smem_raw + C::oCross;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tc::smem_u32(smem_raw) & 1023u) {
    if (tid == 0) flag(p.dev_status, FLARE_DEV_WAIT_TIMEOUT);
    return;
  }
  if (tid == 0) {
    sh.abort_flag = 0;
    for (int s = 0; s < C::kRing; ++s) {
      tc::mbar_init(&sh.full[s], 1);
      tc::mbar_init(&sh.empty[s], kTlCompute);
    }
    tc::mbar_init(&sh.kq_full, 1);
    tc::mbar_init(&sh.v_full, 1);
    tc::mbar_init(&sh.done, kTlCompute);
    tc::mbar_init(&sh.mma_done, 1);
    tc::mbar_init(&sh.upd, 1);
    for (int b = 0; b < 2; ++b) tc::mbar_init(&sh.op_free[b], 1);
    for (int b = 0; b < 3; ++b) tc::mbar_init(&sh.meta_full[b], 1);
    tc::fence_mbar_init();
  }
  if (warp == 4) tc::tmem_alloc(&sh.tmem_base, C::kTmem);
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmS = sh.tmem_base;  // S0^T by pieces, bf16 pairs: 16 columns high, 16 low parts;
                                      // then G, then deltas
  const uint32_t tmW = tmS + C::kTmem - 2 * BM;  // W^T: [K part | Q part], then [X | Y]
  const int total = p.R * p.Hv;

  if (warp == 4) {
    // ------------------------------------------------------------ producer
    const uint32_t idW = tc::idesc_bf16(128, 2 * BM, false, false);
    const uint32_t idG = tc::idesc_bf16(128, BM, false, false);
    if (lane == 0) {
      tc::prefetch_tmap(&maps.k);
      tc::prefetch_tmap(&maps.q);
      tc::prefetch_tmap(&maps.v);
    }
    bool ok = true;
    uint32_t issued = 0;  // ring pieces so far
    int items = 0;        // items whose meta is written
    int kq_items = 0;     // items whose keys and queries are requested
    int v_items = 0;      // items whose values are
    int mma_items = 0;    // items whose MMAs are committed
    int it = blockIdx.x;
    const uint64_t kq_desc = tc::sdesc_sw128(tc::smem_u32(KQ), 16, 1024);

    // The next item with something to do, from `it` on (-1: none), its number
    // of nodes and its slot.
    auto next_item = [&](int& n, int& slot) -> int {
      for (; it < total; it += gridDim.x) {
        const int r = it / p.Hv, j = it - r * p.Hv;
        n = p.node_len[r];
        slot = p.state_slot[r];
        int bad = 0;
        if (n < 0 || n > p.B) bad |= FLARE_DEV_BAD_TREE;
        if (slot < 0 || slot >= p.nslots) bad |= FLARE_DEV_BAD_SLOT;
        if (bad) {
          if (lane == 0) flag(p.dev_status, bad);
        } else if (n == 0) {  // rests this round
          for (int e = lane; e < p.B * (kTlD / 8); e += 32)
            *reinterpret_cast<uint4*>(
                static_cast<__nv_bfloat16*>(p.out_causal) +
                (((size_t)r * p.B + e / (kTlD / 8)) * p.Hv + j) * kTlD + (e % (kTlD / 8)) * 8) =
                make_uint4(0u, 0u, 0u, 0u);
        } else {
          const int found = it;
          it += gridDim.x;
          return found;
        }
      }
      return -1;
    };
    // Its paths and gates into the next meta buffer.
    auto write_meta = [&](int item, int n) {
      TlMeta<BM>& m = sh.meta[items % 3];
      if (item >= 0) {
        const int r = item / p.Hv, j = item - r * p.Hv;
        const size_t g0 = (size_t)r * p.B * p.Hv + j;
        float x0 = lane < n ? tree_log_gate(p.log_decay[g0 + (size_t)lane * p.Hv]) : 0.f;
        float x1 =
            lane + 32 < n ? tree_log_gate(p.log_decay[g0 + (size_t)(lane + 32) * p.Hv]) : 0.f;
        const float b0 = lane < n ? p.beta[g0 + (size_t)lane * p.Hv] : 0.f;
        const float b1 = lane + 32 < n ? p.beta[g0 + (size_t)(lane + 32) * p.Hv] : 0.f;
        int p0, p1;
        if (!warp_load_tree(p.parent + (size_t)r * p.B, n, p0, p1)) {
          if (lane == 0) flag(p.dev_status, FLARE_DEV_BAD_TREE);
          n = -1;
          p0 = p1 = -1;
        }
        uint64_t a0, a1;
        warp_paths<BM>(n, p0, p1, a0, a1, x0, x1);
        if (lane < BM) {
          m.anc[lane] = a0;
          m.gam2[lane] = x0 * 1.4426950408889634f;
          m.beta[lane] = b0;
        }
        if constexpr (BM == 64) {
          m.anc[lane + 32] = a1;
          m.gam2[lane + 32] = x1 * 1.4426950408889634f;
          m.beta[lane + 32] = b1;
        }
        if (lane == 0) m.n = n;
      }
      if (lane == 0) m.item = item;
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&sh.meta_full[items % 3]);
      ++items;
    };
    auto issue_piece = [&](int item, int slot, int q) {
      if (lane == 0) {
        const int s = issued % C::kRing;
        const float* src = p.state_pool + ((size_t)slot * p.Hv + item % p.Hv) * kTlD * kTlD +
                           (size_t)q * kPieceRows * kTlD;
        tc::mbar_expect_tx(&sh.full[s], kPieceBytes);
        tc::bulk_load(ring + s * kPieceBytes, src, kPieceBytes, &sh.full[s]);
      }
      ++issued;
    };
    auto issue_kq = [&](int item) {
      if (lane == 0) {
        const int r = item / p.Hv, h = (item - r * p.Hv) / (p.Hv / p.Hk);
        tc::mbar_expect_tx(&sh.kq_full, C::kKQ);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          tc::tma_load_4d(KQ + c * (2 * BM * 128), &maps.k, &sh.kq_full, c * 64, h, 0, r);
          tc::tma_load_4d(KQ + c * (2 * BM * 128) + BM * 128, &maps.q, &sh.kq_full, c * 64, h, 0,
                          r);
        }
      }
      ++kq_items;
    };

    auto issue_v = [&](int item) {
      if (C::kV == 0) return;
      if (lane == 0) {
        const int r = item / p.Hv, j = item - r * p.Hv;
        uint8_t* dst = smem_raw + C::oV;
        tc::mbar_expect_tx(&sh.v_full, C::kV);
        tc::tma_load_4d(dst, &maps.v, &sh.v_full, 0, j, 0, r);
        tc::tma_load_4d(dst + BM * 128, &maps.v, &sh.v_full, 64, j, 0, r);
      }
      ++v_items;
    };

    // the item at work, the next one and the one after
    int slot = 0, slot_next = 0, n = 0, n_next = 0;
    int cur = next_item(n, slot), nxt = -1;
    if (cur >= 0) {
      for (int q = 0; q < C::kRing; ++q) issue_piece(cur, slot, q);
      issue_kq(cur);
      issue_v(cur);
      write_meta(cur, n);
      nxt = next_item(n_next, slot_next);
      write_meta(nxt, n_next);
    } else {
      write_meta(-1, 0);
    }
    uint32_t used = 0;  // ring pieces consumed
    while (cur >= 0 && ok) {
      // this item's pieces become operands in order; each freed slot takes the
      // piece kRing ahead, this item's or the next one's
      for (int q = 0; q < kPieces && ok; ++q, ++used) {
        const int s = used % C::kRing;
        if (!tl_warp_wait(&sh.empty[s], (used / C::kRing) & 1u, &sh.abort_flag)) {
          ok = false;
          break;
        }
        if (q + C::kRing < kPieces) issue_piece(cur, slot, q + C::kRing);
        else if (nxt >= 0) issue_piece(nxt, slot_next, q + C::kRing - kPieces);
        if (q == 0 && !tl_warp_wait(&sh.kq_full, (uint32_t)(kq_items - 1) & 1u, &sh.abort_flag)) {
          ok = false;
          break;
        }
        tc::fence_after_sync();
        if (tc::elect_one()) {
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            const uint64_t kq =
                kq_desc +
                (uint64_t)(((q >> 1) * (2 * BM * 128) + ((2 * q + kk) & 3) * 32) >> 4);
            const uint32_t op = tmS + q % C::kOps * 32 + kk * 8;
            tc::mma_bf16_ts(tmW, op, kq, idW, q + kk > 0);
            tc::mma_bf16_ts(tmW, op + 16, kq, idW, 1);
          }
          if (q + C::kOps < kPieces) tc::mma_commit(&sh.op_free[q]);
          if (q == kPieces - 1) {
            // G goes over the first pieces' operands: one thread's MMAs execute in
            // issue order, whatever their shapes, so W^T has read them by then
#pragma unroll
            for (int kk = 0; kk < kTlD / 16; ++kk) {
              const uint64_t kd =
                  kq_desc + (uint64_t)(((kk >> 2) * (2 * BM * 128) + (kk & 3) * 32) >> 4);
              tc::mma_bf16_ss(tmS, kd, kd, idG, kk > 0);
            }
            tc::mma_commit(&sh.mma_done);
          }
        }
        __syncwarp();
      }
      if (!ok) break;
      ++mma_items;
      // the next keys and queries at once where the products alone read theirs
      if (!C::kOverlay && nxt >= 0) {
        ok = tl_warp_wait(&sh.mma_done, (uint32_t)(mma_items - 1) & 1u, &sh.abort_flag);
        if (!ok) break;
        issue_kq(nxt);
      }
      // every compute thread is past the previous item: its meta buffer takes
      // the item after the next
      int slot_after = 0, n_after = 0, after = -1;
      if (nxt >= 0) {
        after = next_item(n_after, slot_after);
        write_meta(after, n_after);
        // the values' buffer, and the one that the table shares, once the
        // readout is done
        ok = tl_warp_wait(&sh.done, (uint32_t)(mma_items - 1) & 1u, &sh.abort_flag);
        if (!ok) break;
        tc::fence_async_smem();
        if (C::kOverlay) issue_kq(nxt);
        issue_v(nxt);
      }
      cur = nxt;
      slot = slot_next;
      nxt = after;
      slot_next = slot_after;
    }
    if (!ok && lane == 0 && !sh.abort_flag) {
      sh.abort_flag = 1;
      flag(p.dev_status, FLARE_DEV_WAIT_TIMEOUT);
    }
    __syncwarp();
    if (*reinterpret_cast<volatile int*>(&sh.abort_flag)) {  // let what is in flight land
      for (uint32_t back = 1; back <= C::kRing && back <= issued; ++back) {
        const uint32_t x = issued - back;
        tc::mbar_wait(&sh.full[x % C::kRing], (x / C::kRing) & 1u, nullptr, 100000000ull);
      }
      if (kq_items)
        tc::mbar_wait(&sh.kq_full, (uint32_t)(kq_items - 1) & 1u, nullptr, 100000000ull);
      if (v_items) tc::mbar_wait(&sh.v_full, (uint32_t)(v_items - 1) & 1u, nullptr, 100000000ull);
      __syncwarp();
      if (tc::elect_one()) {
        tc::mma_commit(&sh.mma_done);
        tc::mbar_wait(&sh.mma_done, (uint32_t)mma_items & 1u, nullptr, 100000000ull);
      }
      __syncwarp();
    }
  } else {
    // ------------------------------------------------------------ compute
    const uint32_t lane_off = (uint32_t)(warp * 32) << 16;
    uint32_t used = 0;       // ring pieces consumed
    uint32_t upd_phase = 0;  // of the updates between blocks
    bool bad = false;
    // the k-th item (-1: no more, or a wait that gave up)
    auto take_item = [&](int k) -> int {
      bad |= !tc::mbar_wait(&sh.meta_full[k % 3], (uint32_t)(k / 3) & 1u, &sh.abort_flag);
      const int item = bad ? -1 : sh.meta[k % 3].item;
      return item;
    };
    int item = take_item(0);
#pragma unroll 1
    for (int k = 0;; ++k) {
      const TlMeta<BM>& m = sh.meta[k % 3];
      const int n = m.n;
      if (item < 0) {  // a barrier on this way out too: a thread that gave up
        tl_compute_or(bad);  // meets the others here or at the tables
        break;
      }
      const int r = item / p.Hv, j = item - r * p.Hv;
      const size_t row0 = ((size_t)r * p.B * p.Hv + j) * kTlD;
      const size_t row_stride = (size_t)p.Hv * kTlD;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out_causal) + row0 + (tid & ~1);
      const unsigned short* vs =  // this column's values, 64 elements a row
          reinterpret_cast<const unsigned short*>(smem_raw + C::oV + (tid >> 6) * (BM * 128)) +
          (tid & 63);
      constexpr int kVr = C::kV == 0 ? BM : 1;
      uint32_t vr[kVr];  // BM = 16: this column's values, on their way meanwhile
      if (C::kV == 0) {
        const unsigned short* v = static_cast<const unsigned short*>(p.v) + row0 + tid;
#pragma unroll
        for (int i = 0; i < kVr; ++i) vr[i] = __ldg(v + (size_t)min(i, p.B - 1) * row_stride);
      }
      // the state, piece by piece, into tensor memory as bf16 high and low parts
#pragma unroll 1
      for (int q = 0; q < kPieces; ++q, ++used) {
        const int s = used % C::kRing;
        bad |= !tc::mbar_wait(&sh.full[s], (used / C::kRing) & 1u, &sh.abort_flag);
        __syncwarp();
        const float* S = reinterpret_cast<const float*>(ring + s * kPieceBytes) + tid;
        uint32_t hi[16], lo[16];
#pragma unroll
        for (int e = 0; e < 16; ++e)
          tl_split(S[(2 * e) * kTlD], S[(2 * e + 1) * kTlD], hi[e], lo[e]);
        if (q >= C::kOps) {  // the products with the columns' last piece are through
          bad |= !tc::mbar_wait(&sh.op_free[q - C::kOps], (uint32_t)k & 1u, &sh.abort_flag);
          __syncwarp();
          tc::fence_after_sync();
        }
        const uint32_t op = tmS + lane_off + q % C::kOps * 32;
        tc::tmem_st16(op, hi);
        tc::tmem_st16(op + 16, lo);
        tc::tmem_st_wait();
        tc::fence_before_sync();
        tc::mbar_arrive(&sh.empty[s]);
      }
      bad |= !tc::mbar_wait(&sh.mma_done, (uint32_t)k & 1u, &sh.abort_flag);
      __syncwarp();
      tc::fence_after_sync();
      if (C::kV != 0) bad |= !tc::mbar_wait(&sh.v_full, (uint32_t)k & 1u, &sh.abort_flag);
      __syncwarp();
      auto x_of = [&](int i, uint32_t v, uint32_t w) {
        return m.beta[i] * (__uint_as_float(v << 16) - tc::ex2(m.gam2[i]) * __uint_as_float(w));
      };
      auto y_of = [&](int i, uint32_t w) { return tc::ex2(m.gam2[i]) * __uint_as_float(w); };
      if constexpr (BM > 16) {  // W^T becomes [X | Y], where the blocks' sums gather
#pragma unroll 1
        for (int c0 = 0; c0 < BM; c0 += 16) {
          uint32_t wk[16], wq[16];
          tc::tmem_ld16(tmW + lane_off + c0, wk);
          tc::tmem_ld16(tmW + lane_off + BM + c0, wq);
          tc::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            // unused nodes' rows may hold anything: their sums are not read, and
            // their table rows are zero
            wk[e] = __float_as_uint(x_of(c0 + e, vs[(c0 + e) * 64], wk[e]));
            wq[e] = __float_as_uint(y_of(c0 + e, wq[e]));
          }
          tc::tmem_st16(tmW + lane_off + c0, wk);
          tc::tmem_st16(tmW + lane_off + BM + c0, wq);
        }
        tc::tmem_st_wait();
      }
      // the tables: lane i < BM of G's rows gives -A's row i, lane BM + i M's
      if (warp * 32 < 2 * BM) {
        const bool is_m = tid >= BM;
        const int i = is_m ? tid - BM : tid, own = i >> 4;
        const uint64_t path = m.anc[i];  // empty from n on
        const float gi = m.gam2[i], f = is_m ? 1.f : -m.beta[i];
        const uint64_t see = is_m ? path : path & ~(1ull << i);
#pragma unroll 1
        for (int blk = 0; blk < C::kBlocks; ++blk) {
          uint32_t g[16];
          tc::tmem_ld16(tmS + lane_off + 16 * blk, g);
          tc::tmem_ld_wait();
          float v[16];
          const uint32_t mask = (uint32_t)(see >> (16 * blk));
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const float4 gj = *reinterpret_cast<const float4*>(&m.gam2[16 * blk + 4 * u]);
            const float gv[4] = {gj.x, gj.y, gj.z, gj.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {  // masked by selects: exp may overflow off the path
              const float x = f * tc::ex2(gi - gv[e]) * __uint_as_float(g[4 * u + e]);
              v[4 * u + e] = (mask >> (4 * u + e)) & 1 ? x : 0.f;
            }
          }
          if (blk == own) {
            float* row = Tp + own * 512;
#pragma unroll
            for (int c = 0; c < 16; ++c)
              row[tl_at(i & 15, c >> 1) + 2 * (c & 1) + (is_m ? 1 : 0)] = v[c];
          } else if (blk < own) {
            uint32_t hi[8], lo[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) tl_split(v[2 * c], v[2 * c + 1], hi[c], lo[c]);
            uint8_t* row = Cross + (is_m ? 2 : 0) * C::kCross + (i - 16) * 128;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const int at = ((2 * blk + u) ^ (i & 7)) << 4;
              *reinterpret_cast<uint4*>(row + at) =
                  make_uint4(hi[4 * u], hi[4 * u + 1], hi[4 * u + 2], hi[4 * u + 3]);
              *reinterpret_cast<uint4*>(row + C::kCross + at) =
                  make_uint4(lo[4 * u], lo[4 * u + 1], lo[4 * u + 2], lo[4 * u + 3]);
            }
          }
        }
        if (BM > 16) tc::fence_async_smem();  // the cross tables are MMA operands
      }
      tc::fence_before_sync();
      if (tl_compute_or(bad)) break;  // the tables are complete

      // Rows i, i + 1 of this column and its neighbour: adjacent lanes swap a
      // value, so that each stores a bf16 pair of two columns.
      const bool odd = lane & 1;
      auto store2 = [&](int i, float a, float b) {
        const float recv = __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
        const int row = odd ? i + 1 : i;
        if (row < p.B && n >= 0)
          *reinterpret_cast<uint32_t*>(out + row * row_stride) =
              odd ? tl_pack(recv, b) : tl_pack(a, recv);
      };
      bool out_of_time = false;
#pragma unroll 1
      for (int blk = 0; blk < C::kBlocks; ++blk) {
        const int i0 = 16 * blk;
        if (i0 >= n) {  // unused nodes
          for (int e = 0; e < 16; e += 2) store2(i0 + e, 0.f, 0.f);
          continue;
        }
        const float* T = Tp + blk * 512;
        uint32_t xr[16], yr[16];
        tc::tmem_ld16(tmW + lane_off + i0, xr);
        tc::tmem_ld16(tmW + lane_off + BM + i0, yr);
        tc::tmem_ld_wait();
        uint64_t xy[16];  // {X, Y}, then {delta, the later nodes' share of the readout}
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int i = i0 + e;
          xy[e] = i >= n     ? 0ull
                  : BM == 16 ? f2(x_of(i, vr[e % kVr], xr[e]), y_of(i, yr[e]))
                             : f2(__uint_as_float(xr[e]), __uint_as_float(yr[e]));
        }
        // two nodes a step, their deltas at once into all later nodes' sums
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          float o0 = 0.f, o1 = 0.f;
          if (i0 + 2 * u < n) {
            const float m0 = T[tl_at(2 * u, u) + 1];  // columns 2 u, 2 u + 1 of rows 2 u, ..
            const ulonglong2 c1 = *reinterpret_cast<const ulonglong2*>(T + tl_at(2 * u + 1, u));
            float x, y, m1, unused;
            f2_split(xy[2 * u], x, y);
            const uint64_t d0 = f2_dup(x);
            o0 = p.scale * fmaf(m0, x, y);
            xy[2 * u + 1] = f2_fma(c1.x, d0, xy[2 * u + 1]);
            f2_split(xy[2 * u + 1], x, y);
            f2_split(c1.y, unused, m1);
            const uint64_t d1 = f2_dup(x);
            o1 = p.scale * fmaf(m1, x, y);
#pragma unroll
            for (int e = 2 * u + 2; e < 16; ++e) {
              const ulonglong2 c = *reinterpret_cast<const ulonglong2*>(T + tl_at(e, u));
              xy[e] = f2_fma(c.y, d1, f2_fma(c.x, d0, xy[e]));
            }
          }
          store2(i0 + 2 * u, o0, i0 + 2 * u + 1 < n ? o1 : 0.f);
        }
        if (BM > 16 && i0 + 16 < n) {
          // this block's deltas into the later blocks' sums
          uint32_t hl[16];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float a, b, unused;
            f2_split(xy[2 * e], a, unused);
            f2_split(xy[2 * e + 1], b, unused);
            tl_split(a, b, hl[e], hl[8 + e]);
          }
          tc::tmem_st16(tmS + lane_off, hl);
          tc::tmem_st_wait();
          tc::fence_before_sync();
          tc::named_bar_sync(1, kTlCompute);
          if (warp == 0) {
            tc::fence_after_sync();
            const int rows = BM - 16 - i0;  // of the later blocks
            const uint32_t id = tc::idesc_bf16(128, rows, false, false);
            const uint64_t base = tc::sdesc_sw128(tc::smem_u32(Cross), 16, 1024) +
                                  (uint64_t)((i0 * 128 + blk * 32) >> 4);
            if (tc::elect_one()) {
#pragma unroll
              for (int part = 0; part < 2; ++part) {  // -A into X, M into Y
                const uint32_t d = tmW + part * BM + i0 + 16;
                const uint64_t hi = base + (uint64_t)((2 * part * C::kCross) >> 4);
                const uint64_t lo = hi + (uint64_t)(C::kCross >> 4);
                tc::mma_bf16_ts(d, tmS, hi, id, 1);
                tc::mma_bf16_ts(d, tmS, lo, id, 1);
                tc::mma_bf16_ts(d, tmS + 8, hi, id, 1);
              }
              tc::mma_commit(&sh.upd);
            }
            __syncwarp();
          }
          // after a timeout on: the same barriers, nothing waited for
          if (!out_of_time) out_of_time = !tc::mbar_wait(&sh.upd, upd_phase, &sh.abort_flag);
          upd_phase ^= 1u;
          __syncwarp();
          tc::fence_after_sync();
        }
      }
      bad |= out_of_time;
      tc::fence_before_sync();
      tc::mbar_arrive(&sh.done);
      item = take_item(k + 1);
    }
    if (bad && !sh.abort_flag) {
      sh.abort_flag = 1;
      flag(p.dev_status, FLARE_DEV_WAIT_TIMEOUT);
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 4) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmS, C::kTmem);
  }
}

// ------------------------------------------------------------------ host side

namespace {

PFN_cuTensorMapEncodeTiled_v12000 tl_encode_fn() {
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

// [R, N, H, 128] bf16 as a 4-D map (128, H, N, R), box (64, 1, rows, 1); rows
// past N read as zero
bool tl_map(CUtensorMap* m, const void* x, const GdrParams& p, int H, int rows, bool swizzle) {
  auto fn = tl_encode_fn();
  if (!fn) return false;
  const cuuint64_t gd[4] = {(cuuint64_t)kTlD, (cuuint64_t)H, (cuuint64_t)p.B, (cuuint64_t)p.R};
  const cuuint64_t gs[3] = {(cuuint64_t)kTlD * 2, (cuuint64_t)H * kTlD * 2,
                            (cuuint64_t)p.B * H * kTlD * 2};
  const cuuint32_t bx[4] = {64, 1, (cuuint32_t)rows, 1};
  const cuuint32_t es[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(x), gd, gs, bx, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE,
            swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) ==
         CUDA_SUCCESS;
}

template <int BM>
cudaError_t launch_tl(const GdrParams& p, cudaStream_t stream) {
  TlMaps maps;
  if (!tl_map(&maps.k, p.k, p, p.Hk, BM, true) || !tl_map(&maps.q, p.q, p, p.Hk, BM, true) ||
      !tl_map(&maps.v, p.v, p, p.Hv, BM, false))
    return cudaErrorInvalidValue;
  constexpr int smem = tl_smem<BM>();
  static_assert(TlCfg<BM>::kCtas * (smem + 1024) <= 228 * 1024, "CTAs per SM");
  cudaError_t e = cudaFuncSetAttribute(tree_linear_tc_kernel<BM>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  int dev = 0, sms = kNumSMs;
  if (cudaGetDevice(&dev) == cudaSuccess)
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const long items = (long)p.R * p.Hv, room = (long)TlCfg<BM>::kCtas * sms;
  tree_linear_tc_kernel<BM>
      <<<(unsigned)(items < room ? items : room), kTlThreads, smem, stream>>>(maps, p);
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace

bool tree_linear_tc_supported(int dk, int dv) { return dk == kTlD && dv == kTlD; }

cudaError_t launch_tree_linear_tc(const GdrParams& p, cudaStream_t stream) {
  return p.B <= 16 ? launch_tl<16>(p, stream)
         : p.B <= 32 ? launch_tl<32>(p, stream)
                     : launch_tl<64>(p, stream);
}

}  // namespace flare
