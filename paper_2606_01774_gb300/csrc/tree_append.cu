// KV append of an accepted path: row path[t] of a round's keys and values
// becomes cache position prefix_len + t, for every softmax layer in one launch.
//
// Grid (request, layer): a CTA checks its request's path and pages and copies
// n rows of Hkv heads of both pools in 16-byte pieces, coalesced along the
// head dimension, four pieces in flight per thread.  Bound by launch and
// latency at serving sizes (a round accepts a few tokens per request): 64
// requests, paths of 1 to 8, 12 layers 4.6 us, one request and layer 2.1 us.
#include "common.cuh"
#include "kernels.h"
#include "tree.cuh"

namespace flare {

namespace {
constexpr int kAppendThreads = 256;
}  // namespace

__global__ void __launch_bounds__(kAppendThreads)
    tree_append_kernel(const __grid_constant__ TreeAppendParams p) {
  __shared__ int node[kMaxNodes], page[kMaxNodes], row[kMaxNodes];
  const int r = blockIdx.x, l = blockIdx.y, tid = threadIdx.x;
  const int P = p.prefix_len[r], n = p.path_len[r];
  int bad = 0;
  if (n < 0 || n > p.N) bad = FLARE_DEV_BAD_ACCEPT_LEN;
  else if (P < 0 || (long long)P + n > (long long)p.max_pages * p.page_size)
    bad = FLARE_DEV_BAD_PREFIX_LEN;
  if (!bad && tid < n) {
    const int i = p.path[(size_t)r * p.N + tid];
    const int pg = p.page_table[(size_t)r * p.max_pages + (P + tid) / p.page_size];
    if (i < 0 || i >= p.N) bad |= FLARE_DEV_BAD_TREE;
    if (pg < 0 || pg >= p.num_pages) bad |= FLARE_DEV_BAD_PAGE;
    node[tid] = i;
    page[tid] = pg;
    row[tid] = (P + tid) % p.page_size;
  }
  if (__syncthreads_or(bad)) {
    if (bad && l == 0) flag(p.dev_status, bad);
    return;
  }
  const int row16 = p.D * p.elem_bytes / 16;  // 16-byte pieces per (token, head) row
  const int per_tok = p.Hkv * row16;
  const int total = n * per_tok;  // <= 64 nodes: fits 32 bits for any head count a pool can have
  const uint4* kb = static_cast<const uint4*>(p.k_blk[l]) + (size_t)r * p.N * per_tok;
  const uint4* vb = static_cast<const uint4*>(p.v_blk[l]) + (size_t)r * p.N * per_tok;
  uint4* kp = static_cast<uint4*>(p.k_pool[l]);
  uint4* vp = static_cast<uint4*>(p.v_pool[l]);
  constexpr int kIn = 4;
  for (int e0 = tid; e0 < total; e0 += kIn * kAppendThreads) {
    uint4 kv[kIn], vv[kIn];
    size_t dst[kIn];
#pragma unroll
    for (int u = 0; u < kIn; ++u) {
      const int e = e0 + u * kAppendThreads;
      if (e < total) {
        const int t = e / per_tok, x = e - t * per_tok;  // x = head * row16 + piece
        const int h = x / row16;
        const size_t src = (size_t)node[t] * per_tok + x;
        kv[u] = kb[src];
        vv[u] = vb[src];
        dst[u] = (((size_t)page[t] * p.Hkv + h) * p.page_size + row[t]) * row16 + (x - h * row16);
      }
    }
#pragma unroll
    for (int u = 0; u < kIn; ++u) {
      if (e0 + u * kAppendThreads < total) {
        kp[dst[u]] = kv[u];
        vp[dst[u]] = vv[u];
      }
    }
  }
}

cudaError_t launch_tree_append(const TreeAppendParams& p, cudaStream_t stream) {
  if (p.R == 0) return cudaSuccess;
  tree_append_kernel<<<dim3((unsigned)p.R, (unsigned)p.n_layers), kAppendThreads, 0, stream>>>(p);
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace flare
