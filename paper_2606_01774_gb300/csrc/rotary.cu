// Rotary positions, and the KV append with the rotation on the way.
//
// In a row at position m, pair (a, b) number j of every head becomes
// (a cos t - b sin t, b cos t + a sin t), t = m f_j.  A CTA takes a tile of rows:
// it finds their requests, positions and cache rows, then the cosines and sines
// of its rows once for all heads, then streams the heads through in 32-byte
// units (the two 16-byte pieces that rotate together).  Bound by bytes: every
// element is read and written once.
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

constexpr int kThreads = 256;
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
  for (int i = 1; i < n; ++i) ok = ok && parent[i] >= 0 && parent[i] < i;
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

// Units of a row: heads x (D / 2 Piece::N), the queries', then the keys', then the values'.
template <typename T>
__global__ void __launch_bounds__(kThreads)
    rotary_kernel(const __grid_constant__ RotaryParams p, int tile, int log2_units, int heads) {
  constexpr int N = Piece<T>::N;
  extern __shared__ char smem[];
  float2* turn = reinterpret_cast<float2*>(smem);  // [tile][rd / 2]
  int64_t* pos = reinterpret_cast<int64_t*>(turn + tile * (p.rd / 2));
  int64_t* slot = pos + tile;
  int* live = reinterpret_cast<int*>(slot + tile);
  const int tid = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * tile;
  const int rows = (int)min((int64_t)tile, p.rows - row0);
  const int units = 1 << log2_units, u = tid & (units - 1);
  const int n_q = p.q ? p.Hq : 0, n_k = p.k ? p.Hkv : 0;
  const int pairs = p.rd / 2, turning = p.rd / (2 * N);

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
    const int t = i / pairs;
    if (live[t]) {
      float2 cs = cos_sin((uint64_t)pos[t] * p.table[i - t * pairs]);
      cs.x *= p.amplitude;
      cs.y *= p.inverse ? -p.amplitude : p.amplitude;
      turn[i] = cs;
    }
  }
  __syncthreads();

  // this thread's pieces of a head, in elements, and its pairs
  const bool turns = u < turning;
  const int e0 = !turns || p.interleaved ? 2 * N * u : N * u;
  const int e1 = turns && !p.interleaved ? p.rd / 2 + N * u : e0 + N;
  const int step = kThreads >> log2_units;
  const int total = rows * heads;
  for (int i0 = tid >> log2_units; i0 < total; i0 += step * kUnroll) {
    uint4 a[kUnroll], b[kUnroll];
    int t[kUnroll], h[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const int i = i0 + j * step;
      t[j] = i / heads;
      h[j] = i - t[j] * heads;
      if (i >= total || !live[t[j]]) {
        t[j] = -1;
        continue;
      }
      const int64_t row = row0 + t[j];
      const T* src;
      if (h[j] < n_q) src = static_cast<const T*>(p.q) + row * p.q_stride + h[j] * p.D;
      else if (h[j] < n_q + n_k)
        src = static_cast<const T*>(p.k) + row * p.k_stride + (h[j] - n_q) * p.D;
      else src = static_cast<const T*>(p.v) + row * p.v_stride + (h[j] - n_q - n_k) * p.D;
      a[j] = *reinterpret_cast<const uint4*>(src + e0);
      b[j] = *reinterpret_cast<const uint4*>(src + e1);
    }
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      if (t[j] < 0) continue;
      const int64_t row = row0 + t[j];
      if (turns && h[j] < n_q + n_k) {
        float x[2 * N];
        Piece<T>::load(a[j], x);
        Piece<T>::load(b[j], x + N);
        const float2* cs = turn + t[j] * pairs + N * u;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float2 c = cs[e];
          float& lo = p.interleaved ? x[2 * e] : x[e];
          float& hi = p.interleaved ? x[2 * e + 1] : x[N + e];
          const float y = lo * c.x - hi * c.y;
          hi = hi * c.x + lo * c.y;
          lo = y;
        }
        a[j] = Piece<T>::store(x);
        b[j] = Piece<T>::store(x + N);
      }
      const auto put = [&](void* to, int64_t at) {
        T* dst = static_cast<T*>(to) + at;
        *reinterpret_cast<uint4*>(dst + e0) = a[j];
        *reinterpret_cast<uint4*>(dst + e1) = b[j];
      };
      if (h[j] < n_q) {
        put(p.q_out, row * p.q_out_stride + h[j] * p.D);
      } else if (h[j] < n_q + n_k) {
        const int hk = h[j] - n_q;
        if (p.k_out) put(p.k_out, row * p.k_out_stride + hk * p.D);
        if (p.k_pool) put(p.k_pool, (slot[t[j]] + (int64_t)hk * p.page_size) * p.D);
      } else {
        put(p.v_pool, (slot[t[j]] + (int64_t)(h[j] - n_q - n_k) * p.page_size) * p.D);
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
  int tile = 16;
  while (tile > 1 && (p.rows + tile - 1) / tile < 2 * num_sms) tile /= 2;
  const int smem = tile * (p.rd / 2 * (int)sizeof(float2) + 2 * (int)sizeof(int64_t) +
                           (int)sizeof(int));
  const unsigned grid = (unsigned)((p.rows + tile - 1) / tile);
  rotary_kernel<T><<<grid, kThreads, smem, stream>>>(p, tile, log2_units, heads);
  note_launches(1);
  return cudaGetLastError();
}

cudaError_t launch_rotary(const RotaryParams& p, bool bf16, int num_sms, cudaStream_t stream) {
  if (p.rows == 0 || p.R == 0) return cudaSuccess;
  return bf16 ? launch<__nv_bfloat16>(p, num_sms, stream) : launch<float>(p, num_sms, stream);
}

}  // namespace flare
