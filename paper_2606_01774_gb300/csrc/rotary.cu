// Rotary positions, and the KV append with the rotation on the way.
//
// In a row at position m, pair (a, b) number j of every head becomes
// (a cos t - b sin t, b cos t + a sin t), t = m f_j.  A CTA takes a tile of rows:
// it finds their requests, positions and cache rows, then the cosines and sines
// of its rows once for all heads, then streams the heads through in 32-byte
// units (the two 16-byte pieces that rotate together).  Bound by bytes: every
// element is read and written once (32768 rows of 9 KiB in bf16: 99 us, 6.1 TB/s, a
// copy's rate being 6.8; prompts appended to pages of 16 with their queries: 61 us,
// 5.8 TB/s).  A few tokens take 3 us, most of it the round trips to memory from
// lengths to positions to table.  Small CTAs, six an SM, so that some stream while
// others work out angles (CTAs of 64, 256 or 512 threads: 4 to 15% slower).
//
// Angles: the table holds f_j as fractions of a turn in 64-bit fixed point, so
// m f_j modulo a turn is one wrapping integer product, exact in the table's
// values at every position; what is left after the nearest quarter turn goes to
// fp32, at most an eighth of a turn, which sincospi takes without a reduction.
#include "common.cuh"
#include "kernels.h"
#include "piece.cuh"

namespace flare {

namespace {

constexpr int kThreads = 128;
constexpr int kCtas = 6;     // of an SM
constexpr int kTileBytes = 48 << 10;
constexpr int kUnroll = 4;  // units in flight per thread

// cos and sin of `phase` / 2^64 turns.
__device__ __forceinline__ float2 cos_sin(uint64_t phase) {
  const uint64_t quarter = (phase + (1ull << 61)) >> 62;
  const float rest = (float)(int32_t)(uint32_t)((phase - (quarter << 62)) >> 32);
  float s, c;
  sincospif(rest * 0x1p-31f, &s, &c);
  switch (quarter & 3) {
    case 0: return make_float2(c, s);
    case 1: return make_float2(-s, c);
    case 2: return make_float2(-c, -s);
    default: return make_float2(s, -c);
  }
}

// Depth of node t in a request's tree; -1 when the tree is wrong.
__device__ __forceinline__ int node_depth(const int32_t* __restrict__ parent, int n, int t) {
  bool ok = parent[0] == -1;
#pragma unroll 8
  for (int i = 1; i < n; ++i) ok &= (uint32_t)parent[i] < (uint32_t)i;
  if (!ok) return -1;
  int depth = 0;
  for (int i = t; i > 0; i = parent[i]) ++depth;
  return depth;
}

// Whether row `row` is a token to be handled; its position and, for an append, the
// index of its first head's row in the pools.
__device__ __forceinline__ bool resolve(const RotaryParams& p, int64_t row, int64_t& pos,
                                        int64_t& slot) {
  int r, t, n;
  if (p.token_start) {
    int lo = 0, hi = p.R;  // the last request that starts at or before the row
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.token_start[mid] <= row) lo = mid;
      else hi = mid;
    }
    r = lo;
    const int first = p.token_start[r], last = p.token_start[r + 1];
    if (first < 0 || last > p.rows || first > row || last <= row) return false;
    t = (int)row - first;
    n = last - first;
  } else {
    r = (int)(row / p.B);
    t = (int)(row - (int64_t)r * p.B);
    n = p.token_len ? p.token_len[r] : p.B;
    if (n < 0 || n > p.B) {
      flag(p.dev_status, FLARE_DEV_BAD_ACCEPT_LEN);
      return false;
    }
    if (t >= n) return false;
  }
  const int P = p.prefix_len ? p.prefix_len[r] : 0;
  if (P < 0 || (p.k_pool && (int64_t)P + n > (int64_t)p.max_pages * p.page_size)) {
    flag(p.dev_status, FLARE_DEV_BAD_PREFIX_LEN);
    return false;
  }
  pos = (int64_t)P + t;
  if (p.parent) {
    const int depth = node_depth(p.parent + (size_t)r * p.B, n, t);
    if (depth < 0) {
      flag(p.dev_status, FLARE_DEV_BAD_TREE);
      return false;
    }
    pos = (int64_t)P + depth;
  }
  if (p.k_pool) {
    const int at = P + t;
    const int page = p.page_table[(size_t)r * p.max_pages + at / p.page_size];
    if (page < 0 || page >= p.num_pages) {
      flag(p.dev_status, FLARE_DEV_BAD_PAGE);
      return false;
    }
    slot = (int64_t)page * p.Hkv * p.page_size + at % p.page_size;
  }
  if (p.position) pos = p.position[row];
  return true;
}

}  // namespace

// A head is units of 32 bytes, D / 2N of them (N elements to a piece).  A thread has one unit number
// of every head_slots'th head of a row, so its cosines and sines stay in registers
// from the first head to the last; the CTA takes 128 / (units head_slots) rows at a time.
template <typename T, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads, kCtas)
    rotary_kernel(const __grid_constant__ RotaryParams p, int tile, int log2_units,
                  int log2_slots) {
  constexpr int N = Piece<T>::N;
  extern __shared__ __align__(16) char smem[];
  const int pairs = p.rd / 2, turning = p.rd / (2 * N);
  // [tile][N / 2][turning] {cos, sin, cos, sin}: a unit's pairs two by two, neighbouring units
  // next to each other
  float4* turn = reinterpret_cast<float4*>(smem);
  int64_t* pos = reinterpret_cast<int64_t*>(turn + tile * (pairs / 2));
  int64_t* slot = pos + tile;
  int* live = reinterpret_cast<int*>(slot + tile);
  const int tid = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * tile;
  const int rows = (int)min((int64_t)tile, p.rows - row0);

  if (blockIdx.x == 0 && p.token_start) {
    int bad = 0;
    for (int i = tid; i <= p.R; i += kThreads)
      bad |= p.token_start[i] < 0 || p.token_start[i] > p.rows ||
             (i < p.R && p.token_start[i] > p.token_start[i + 1]);
    if (bad) flag(p.dev_status, FLARE_DEV_BAD_ACCEPT_LEN);
  }
  if (tid < rows) live[tid] = resolve(p, row0 + tid, pos[tid], slot[tid]);
  __syncthreads();
  for (int i = tid; i < rows * pairs; i += kThreads) {
    const int t = i / pairs, j = i - t * pairs, unit = j / N, e = j - unit * N;
    if (live[t]) {
      float2 cs = cos_sin((uint64_t)pos[t] * p.table[j]);
      cs.x *= p.amplitude;
      cs.y *= p.inverse ? -p.amplitude : p.amplitude;
      reinterpret_cast<float2*>(turn + (t * (N / 2) + e / 2) * turning + unit)[e & 1] = cs;
    }
  }
  __syncthreads();

  const int u = tid & ((1 << log2_units) - 1), row_threads = log2_units + log2_slots;
  const int first = (tid >> log2_units) & ((1 << log2_slots) - 1), slots = 1 << log2_slots;
  const int n_q = p.q ? p.Hq : 0, n_k = n_q + (p.k ? p.Hkv : 0);
  const int heads = n_k + (p.k_pool ? p.Hkv : 0);
  // this thread's pieces of a head, in elements
  const bool turns = u < turning;
  const int e0 = !turns || INTERLEAVED ? 2 * N * u : N * u;
  const int e1 = turns && !INTERLEAVED ? pairs + N * u : e0 + N;
  for (int t = tid >> row_threads; t < rows; t += kThreads >> row_threads) {
    if (!live[t]) continue;
    float c[N], s[N];
    if (turns) {
#pragma unroll
      for (int k = 0; k < N / 2; ++k) {
        const float4 f = turn[(t * (N / 2) + k) * turning + u];
        c[2 * k] = f.x, s[2 * k] = f.y, c[2 * k + 1] = f.z, s[2 * k + 1] = f.w;
      }
    }
    const int64_t row = row0 + t;
    const T* q = static_cast<const T*>(p.q) + row * p.q_stride;
    const T* k = static_cast<const T*>(p.k) + row * p.k_stride - n_q * p.D;
    const T* v = static_cast<const T*>(p.v) + row * p.v_stride - n_k * p.D;
    T* q_out = static_cast<T*>(p.q_out) + row * p.q_out_stride;
    T* k_out = static_cast<T*>(p.k_out) + row * p.k_out_stride - n_q * p.D;
    const int64_t pool_head = (int64_t)p.page_size * p.D;
    for (int h0 = first; h0 < heads; h0 += slots * kUnroll) {
      uint4 a[kUnroll], b[kUnroll];
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) {
        const int h = h0 + j * slots;
        if (h < heads) {
          const T* src = (h < n_q ? q : h < n_k ? k : v) + h * p.D;
          a[j] = *reinterpret_cast<const uint4*>(src + e0);
          b[j] = *reinterpret_cast<const uint4*>(src + e1);
        }
      }
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) {
        const int h = h0 + j * slots;
        if (h >= heads) continue;
        if (turns && h < n_k) {
          float x[2 * N];
          Piece<T>::load(a[j], x);
          Piece<T>::load(b[j], x + N);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            float& lo = x[INTERLEAVED ? 2 * e : e];
            float& hi = x[INTERLEAVED ? 2 * e + 1 : N + e];
            const float y = lo * c[e] - hi * s[e];
            hi = hi * c[e] + lo * s[e];
            lo = y;
          }
          a[j] = Piece<T>::store(x);
          b[j] = Piece<T>::store(x + N);
        }
        const auto put = [&](T* dst) {
          *reinterpret_cast<uint4*>(dst + e0) = a[j];
          *reinterpret_cast<uint4*>(dst + e1) = b[j];
        };
        if (h < n_q) {
          put(q_out + h * p.D);
        } else if (h < n_k) {
          if (p.k_out) put(k_out + h * p.D);
          if (p.k_pool)
            put(static_cast<T*>(p.k_pool) + slot[t] * p.D + (h - n_q) * pool_head);
        } else {
          put(static_cast<T*>(p.v_pool) + slot[t] * p.D + (h - n_k) * pool_head);
        }
      }
    }
  }
}

__global__ void rotary_table_kernel(const flare_rotary_freq_desc d, uint64_t* table) {
  const int j = threadIdx.x;
  if (2 * j >= d.rotary_dim) return;
  constexpr double kTwoPi = 6.283185307179586476925;
  double base = d.base;
  if (d.scaling == FLARE_ROTARY_BASE)
    base *= pow(d.factor, (double)d.rotary_dim / (d.rotary_dim - 2));
  double f = pow(base, -2.0 * j / d.rotary_dim);
  if (d.scaling == FLARE_ROTARY_LINEAR) f /= d.factor;
  if (d.scaling == FLARE_ROTARY_BY_PARTS) {
    const double turns = d.original_len * f / kTwoPi;
    const double keep =
        fmin(fmax((turns - d.low_turns) / (d.high_turns - d.low_turns), 0.0), 1.0);
    f = keep * f + (1.0 - keep) * f / d.factor;
  }
  const double turn = f / kTwoPi;
  table[j] = (uint64_t)((turn - floor(turn)) * 0x1p64);
}

cudaError_t launch_rotary_table(const flare_rotary_freq_desc& d, uint64_t* table,
                                cudaStream_t stream) {
  rotary_table_kernel<<<1, 128, 0, stream>>>(d, table);
  note_launches(1);
  return cudaGetLastError();
}

template <typename T>
static cudaError_t launch(const RotaryParams& p, int num_sms, cudaStream_t stream) {
  int log2_units = 0;
  while ((2 * Piece<T>::N << log2_units) < p.D) ++log2_units;
  const int heads = (p.q ? p.Hq : 0) + (p.k ? p.Hkv : 0) + (p.k_pool ? p.Hkv : 0);
  // tiles of up to 48 KiB: larger ones leave a CTA's memory idle while it works out its next angles
  // (32768 rows of 9 KiB: 117 us with 32 rows, 110 with 16, 105 with 8, 99 with 4, 101 with
  // 2), smaller ones work out few at a time (of 6 KiB: 63, 61, 61, 62, 67)
  int tile = 16;
  const auto tiles = [&] { return ((int64_t)p.rows + tile - 1) / tile; };
  while (tile > 1 && ((int64_t)tile * heads * p.D * (int)sizeof(T) > kTileBytes ||
                      tiles() < 2 * num_sms))
    tile /= 2;
  // as many rows at a time as the tile has, or four heads in flight per thread
  int log2_slots = 0;
  while (log2_units + log2_slots < 7 && (tile << (log2_units + log2_slots) < kThreads ||
                                         heads >> log2_slots > kUnroll))
    ++log2_slots;
  const int smem = tile * (p.rd / 4 * (int)sizeof(float4) + 2 * (int)sizeof(int64_t) +
                           (int)sizeof(int));
  const unsigned grid = (unsigned)tiles();
  if (p.interleaved)
    rotary_kernel<T, true><<<grid, kThreads, smem, stream>>>(p, tile, log2_units, log2_slots);
  else
    rotary_kernel<T, false><<<grid, kThreads, smem, stream>>>(p, tile, log2_units, log2_slots);
  note_launches(1);
  return cudaGetLastError();
}

cudaError_t launch_rotary(const RotaryParams& p, bool bf16, int num_sms, cudaStream_t stream) {
  if (p.rows == 0 || p.R == 0) return cudaSuccess;
  return bf16 ? launch<__nv_bfloat16>(p, num_sms, stream) : launch<float>(p, num_sms, stream);
}

}  // namespace flare
