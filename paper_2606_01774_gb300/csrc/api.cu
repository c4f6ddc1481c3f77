// C ABI of the FLARE attention step: argument checks, work planning, launch.
// The declarations and the contract of every entry point are in flare.h.
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <atomic>
#include <initializer_list>

#include "flare.h"
#include "kernels.h"

using namespace flare;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

bool valid_dtype(flare_dtype d) { return d == FLARE_DT_BF16 || d == FLARE_DT_F32; }

flare_status check_linear(const flare_linear_desc* d) {
  if (!d) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests < 0 || d->block_len < 1 || d->num_qk_heads < 1 || d->num_v_heads < 1 ||
      d->num_state_slots < 1 || !valid_dtype(d->act_dtype))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_v_heads % d->num_qk_heads != 0) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->block_len > 64) return FLARE_ERR_UNSUPPORTED;
  if ((d->head_dim_k != 64 && d->head_dim_k != 128) ||
      (d->head_dim_v != 64 && d->head_dim_v != 128))
    return FLARE_ERR_UNSUPPORTED;
  return FLARE_OK;
}

flare_status check_softmax(const flare_softmax_desc* d) {
  if (!d) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests < 0 || d->block_len < 1 || d->num_q_heads < 1 || d->num_kv_heads < 1 ||
      d->page_size < 1 || d->num_pages < 0 || d->max_pages_per_req < 0 ||
      !valid_dtype(d->act_dtype))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->mask_mode != FLARE_MASK_BLOCK_BIDIR && d->mask_mode != FLARE_MASK_BLOCK_CAUSAL &&
      d->mask_mode != FLARE_MASK_ROW_TYPE_UNIFORM &&
      d->mask_mode != FLARE_MASK_ROW_TYPE_PER_REQUEST)
    return FLARE_ERR_INVALID_ARGUMENT;
  if ((d->mask_mode == FLARE_MASK_ROW_TYPE_UNIFORM ||
       d->mask_mode == FLARE_MASK_ROW_TYPE_PER_REQUEST) && !d->row_type)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!(d->scale >= 0.f) || !(d->scale < 3.0e38f)) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_q_heads % d->num_kv_heads != 0) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->block_len > 64) return FLARE_ERR_UNSUPPORTED;
  if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256) return FLARE_ERR_UNSUPPORTED;
  if (d->page_size != 16 && d->page_size != 32 && d->page_size != 64 && d->page_size != 128)
    return FLARE_ERR_UNSUPPORTED;
  if ((int64_t)d->max_pages_per_req * d->page_size > (1 << 24)) return FLARE_ERR_UNSUPPORTED;
  return FLARE_OK;
}

int device_sms() {
  int dev = 0, n = kNumSMs;
  if (cudaGetDevice(&dev) == cudaSuccess)
    cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
  return n > 0 ? n : kNumSMs;
}

SoftmaxParams softmax_params(const flare_softmax_desc* d) {
  SoftmaxParams p;
  memset(&p, 0, sizeof p);
  p.R = d->num_requests;
  p.B = d->block_len;
  p.Hq = d->num_q_heads;
  p.Hkv = d->num_kv_heads;
  p.G = d->num_q_heads / d->num_kv_heads;
  p.D = d->head_dim;
  p.page_size = d->page_size;
  p.num_pages = d->num_pages;
  p.max_pages = d->max_pages_per_req;
  p.scale_log2 = d->scale * 1.4426950408889634f;
  p.causal = d->mask_mode == FLARE_MASK_BLOCK_CAUSAL;
  if (d->mask_mode == FLARE_MASK_ROW_TYPE_UNIFORM || d->mask_mode == FLARE_MASK_ROW_TYPE_PER_REQUEST) {
    p.row_type = d->row_type;
    p.row_type_stride = d->mask_mode == FLARE_MASK_ROW_TYPE_PER_REQUEST ? d->block_len : 0;
  }
  return p;
}

SoftmaxPlan plan_for(const flare_softmax_desc* d) {
  return plan_softmax(d->num_requests, d->block_len, d->num_q_heads, d->num_kv_heads,
                      d->head_dim, d->page_size, d->max_pages_per_req,
                      d->act_dtype == FLARE_DT_BF16, device_sms());
}

// The tree calls read no mask fields of a softmax descriptor.
flare_status check_tree_softmax(const flare_softmax_desc* d) {
  if (!d) return FLARE_ERR_INVALID_ARGUMENT;
  flare_softmax_desc t = *d;
  t.mask_mode = FLARE_MASK_BLOCK_BIDIR;
  t.row_type = nullptr;
  return check_softmax(&t);
}

TreeSoftmaxPlan tree_plan_for(const flare_softmax_desc* d) {
  return plan_tree_softmax(d->num_requests, d->block_len, d->num_q_heads, d->num_kv_heads,
                           d->head_dim, d->page_size, d->max_pages_per_req,
                           d->act_dtype == FLARE_DT_BF16, device_sms());
}

flare_status check_tree_verify(const flare_tree_verify_desc* d) {
  if (!d) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests < 0 || d->num_nodes < 1 || d->vocab_size < 1 ||
      !valid_dtype(d->logits_dtype) ||
      (d->mode != FLARE_VERIFY_GREEDY && d->mode != FLARE_VERIFY_SAMPLE))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->mode == FLARE_VERIFY_SAMPLE &&
      (!(d->inv_temperature > 0.f) || !(d->inv_temperature < 3.0e38f)))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_nodes > 64 || d->vocab_size > (1 << 24)) return FLARE_ERR_UNSUPPORTED;
  return FLARE_OK;
}

bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

// Whether the byte ranges of two arrays share a byte.
bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + b_bytes && y < x + a_bytes;
}

size_t elem_bytes(flare_dtype d) { return d == FLARE_DT_BF16 ? 2 : 4; }

// Bytes from the first row of an array to the end of its last.
size_t span_bytes(int64_t rows, int64_t stride, int64_t width, size_t elem) {
  return rows > 0 ? (size_t)((rows - 1) * stride + width) * elem : 0;
}

// Rows of an array: `width` elements each, `stride` apart.
struct Rows {
  const void* at;
  int64_t stride, width;
};

// Whether two arrays of `rows` rows share an element.  Rows of the same stride may lie between each
// other, as slices of one projection do.
bool rows_overlap(const Rows& a, const Rows& b, int64_t rows, size_t elem) {
  if (!a.at || !b.at || !overlap(a.at, span_bytes(rows, a.stride, a.width, elem), b.at,
                                 span_bytes(rows, b.stride, b.width, elem)))
    return false;
  if (a.stride != b.stride) return true;
  const int64_t step = a.stride * (int64_t)elem;
  int64_t off = (int64_t)((intptr_t)b.at - (intptr_t)a.at) % step;
  if (off < 0) off += step;
  return off < a.width * (int64_t)elem || off + b.width * (int64_t)elem > step;
}

// Whether every output is clear of the other outputs and of every input, unless it takes an
// input's very place: then each element is read before it is written, by the same thread.
// `own` (rotary): the only input whose place output i may take is the i-th.
bool outputs_clear(const Rows* in, int n_in, const Rows* out, int n_out, bool own, int64_t rows,
                   size_t elem) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j) {
      const bool same = in[j].at == out[i].at && in[j].stride == out[i].stride &&
                        in[j].width == out[i].width && (!own || i == j);
      if (!same && rows_overlap(in[j], out[i], rows, elem)) return false;
    }
    for (int j = 0; j < i; ++j)
      if (rows_overlap(out[j], out[i], rows, elem)) return false;
  }
  return true;
}

bool aligned4(std::initializer_list<const void*> arrays) {
  for (const void* p : arrays)
    if (!aligned(p, 4)) return false;
  return true;
}

flare_status check_rotary(const flare_rotary_desc* d, bool packed, bool append) {
  if (!d) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests < 0 || (packed ? d->num_tokens < 0 : d->block_len < 1) ||
      d->num_q_heads < 1 || d->num_kv_heads < 1 || !valid_dtype(d->act_dtype) ||
      (d->layout != FLARE_ROTARY_HALF && d->layout != FLARE_ROTARY_INTERLEAVED) ||
      (d->inverse != 0 && d->inverse != 1) ||
      !(d->amplitude > -3.0e38f && d->amplitude < 3.0e38f))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256) return FLARE_ERR_UNSUPPORTED;
  if (d->rotary_dim < 16 || d->rotary_dim > d->head_dim || d->rotary_dim % 16)
    return FLARE_ERR_UNSUPPORTED;
  if (d->num_q_heads > 65536 || d->num_kv_heads > 65536) return FLARE_ERR_UNSUPPORTED;
  if (!packed && (int64_t)d->num_requests * d->block_len > INT32_MAX) return FLARE_ERR_UNSUPPORTED;
  const int64_t strides[3] = {d->q_stride, d->k_stride, d->v_stride};
  for (int i = 0; i < 3; ++i) {
    const int64_t width = (int64_t)(i ? d->num_kv_heads : d->num_q_heads) * d->head_dim;
    if (strides[i] && (strides[i] < width || strides[i] * elem_bytes(d->act_dtype) % 16))
      return FLARE_ERR_INVALID_ARGUMENT;
    if (strides[i] > ((int64_t)1 << 31)) return FLARE_ERR_UNSUPPORTED;
  }
  if (append) {
    if (d->page_size < 1 || d->num_pages < 0 || d->max_pages_per_req < 0)
      return FLARE_ERR_INVALID_ARGUMENT;
    if (d->page_size != 16 && d->page_size != 32 && d->page_size != 64 && d->page_size != 128)
      return FLARE_ERR_UNSUPPORTED;
    if ((int64_t)d->max_pages_per_req * d->page_size > (1 << 24)) return FLARE_ERR_UNSUPPORTED;
  }
  return FLARE_OK;
}

bool no_rows(const flare_rotary_desc* d, bool packed) {
  return d->num_requests == 0 || (packed && d->num_tokens == 0);
}

// The rotation of both calls; k_pool is null without an append.
flare_status rotary(const flare_rotary_desc* d, const void* q, const void* k, const void* v,
                    const uint64_t* table, const int32_t* position, const int32_t* prefix_len,
                    const int32_t* token_len, const int32_t* parent, const int32_t* token_start,
                    const int32_t* page_table, void* q_out, void* k_out, void* k_pool,
                    void* v_pool, int32_t* dev_status, void* stream) {
  const int64_t rows =
      token_start ? d->num_tokens : (int64_t)d->num_requests * d->block_len;
  RotaryParams p;
  memset(&p, 0, sizeof p);
  p.R = d->num_requests;
  p.B = d->block_len;
  p.rows = (int)rows;
  p.Hq = d->num_q_heads;
  p.Hkv = d->num_kv_heads;
  p.D = d->head_dim;
  p.rd = d->rotary_dim;
  p.interleaved = d->layout == FLARE_ROTARY_INTERLEAVED;
  p.inverse = d->inverse;
  p.page_size = d->page_size;
  p.num_pages = d->num_pages;
  p.max_pages = d->max_pages_per_req;
  p.amplitude = d->amplitude;
  const int64_t q_width = (int64_t)p.Hq * p.D, k_width = (int64_t)p.Hkv * p.D;
  p.q_stride = d->q_stride ? d->q_stride : q_width;
  p.k_stride = d->k_stride ? d->k_stride : k_width;
  p.v_stride = d->v_stride ? d->v_stride : k_width;
  p.q_out_stride = q_out == q ? p.q_stride : q_width;
  p.k_out_stride = k_out == k ? p.k_stride : k_width;
  const size_t e = elem_bytes(d->act_dtype);
  const Rows in[3] = {{q, p.q_stride, q_width}, {k, p.k_stride, k_width}, {v, p.v_stride, k_width}};
  const Rows out[2] = {{q_out, p.q_out_stride, q_width}, {k_out, p.k_out_stride, k_width}};
  if (!outputs_clear(in, 3, out, 2, true, rows, e) ||
      !aligned4({position, prefix_len, token_len, parent, token_start, page_table, dev_status}))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (k_pool) {
    const size_t pool = (size_t)p.num_pages * p.Hkv * p.page_size * p.D * e;
    for (const Rows& r : {in[0], in[1], in[2], out[0], out[1]}) {
      const size_t bytes = r.at ? span_bytes(rows, r.stride, r.width, e) : 0;
      if (overlap(r.at, bytes, k_pool, pool) || overlap(r.at, bytes, v_pool, pool))
        return FLARE_ERR_INVALID_ARGUMENT;
    }
    if (overlap(k_pool, pool, v_pool, pool)) return FLARE_ERR_INVALID_ARGUMENT;
  }
  p.q = q;
  p.k = k;
  p.v = v;
  p.table = table;
  p.position = position;
  p.prefix_len = prefix_len;
  p.token_len = token_len;
  p.parent = parent;
  p.token_start = token_start;
  p.page_table = page_table;
  p.q_out = q_out;
  p.k_out = k_out;
  p.k_pool = k_pool;
  p.v_pool = v_pool;
  p.dev_status = dev_status;
  const cudaError_t err = launch_rotary(p, d->act_dtype == FLARE_DT_BF16, device_sms(),
                                        static_cast<cudaStream_t>(stream));
  return err == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status check_block_norm(const flare_block_norm_desc* d) {
  if (!d) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_tokens < 0 || d->width < 1 || d->group < 0 || !valid_dtype(d->act_dtype) ||
      (d->shared_weight != 0 && d->shared_weight != 1) ||
      (d->post_norm != 0 && d->post_norm != 1) || (d->pre_norm != 0 && d->pre_norm != 1) ||
      (d->gate_act != FLARE_ACT_NONE && d->gate_act != FLARE_ACT_SILU &&
       d->gate_act != FLARE_ACT_SIGMOID) ||
      !(d->eps > 0.f && d->eps < 3.0e38f) ||
      !(d->residual_scale > -3.0e38f && d->residual_scale < 3.0e38f))
    return FLARE_ERR_INVALID_ARGUMENT;
  const int64_t strides[2] = {d->x_stride, d->gate_stride};
  for (int64_t s : strides) {
    if (s && (s < d->width || s * elem_bytes(d->act_dtype) % 16)) return FLARE_ERR_INVALID_ARGUMENT;
    if (s > ((int64_t)1 << 31)) return FLARE_ERR_UNSUPPORTED;
  }
  if (d->width % 8 || d->width > 16384) return FLARE_ERR_UNSUPPORTED;
  if (d->group && d->group != d->width) {
    if (d->group != 64 && d->group != 128 && d->group != 256) return FLARE_ERR_UNSUPPORTED;
    if (d->width % d->group) return FLARE_ERR_INVALID_ARGUMENT;
  }
  return FLARE_OK;
}

BlockNormParams block_norm_params(const flare_block_norm_desc* d, const void* x, const void* gate,
                                  const void* residual, const float* post_weight,
                                  const float* pre_weight) {
  BlockNormParams p;
  memset(&p, 0, sizeof p);
  p.T = d->num_tokens;
  p.W = d->width;
  p.G = d->group ? d->group : d->width;
  p.shared = d->shared_weight && p.G < d->width;  // of one group the weight has W entries either way
  p.post = d->post_norm;
  p.pre = d->pre_norm;
  p.act = d->gate_act;
  p.eps = d->eps;
  p.alpha = d->residual_scale;
  p.x_stride = d->x_stride ? d->x_stride : d->width;
  p.gate_stride = d->gate_stride ? d->gate_stride : d->width;
  p.x = x;
  p.gate = gate;
  p.residual = residual;
  p.wpost = d->post_norm ? post_weight : nullptr;
  p.wpre = d->pre_norm ? pre_weight : nullptr;
  return p;
}

// Bytes of row statistics, with the cut of a row into chunks.
size_t tree_verify_workspace(const flare_tree_verify_desc* d, int* chunk, int* n_chunks) {
  plan_tree_verify(d->num_requests, d->num_nodes, d->vocab_size, device_sms(), chunk, n_chunks);
  return (size_t)d->num_requests * d->num_nodes * *n_chunks * sizeof(float4);
}

}  // namespace

namespace flare {

static std::atomic<uint64_t> g_launches{0};
void note_launches(int n) { g_launches.fetch_add((uint64_t)n, std::memory_order_relaxed); }

SoftmaxPlan plan_softmax(int R, int B, int Hq, int Hkv, int D, int page_size, int max_pages,
                         bool bf16, int num_sms) {
  SoftmaxPlan pl;
  memset(&pl, 0, sizeof pl);
  const int G = Hq / Hkv, M = B * G;
  const long prefix_max = (long)max_pages * page_size;
  if (bf16 && softmax_tc_supported(B, Hq, Hkv, D, page_size)) {
    // tensor-core kernel: 128 query rows per CTA, one CTA per SM, work units
    // started longest first.  Split the prefix only when the batch has fewer
    // work items than SMs (then aim at two CTAs per SM), and keep at least 16
    // tiles (1024 keys) per split so partials stay small.
    pl.kernel = 1;
    pl.rows_per_cta = 128;
    const long items = (long)R * Hkv * ((M + 127) / 128);
    const long tiles = (prefix_max + 63) / 64;
    long ns = 1;
    if (items > 0 && items < num_sms) ns = (2L * num_sms + items - 1) / items;
    const long cap = tiles / 16 > 1 ? tiles / 16 : 1;
    if (ns > cap) ns = cap;
    if (ns > 64) ns = 64;  // the merge keeps 128 x n_split weights in shared memory
    const long tps = ns > 0 ? (tiles + ns - 1) / ns : 1;
    pl.split_len = (int)((tps > 0 ? tps : 1) * 64);
    pl.n_split = tiles > 0 ? (int)((tiles + tps - 1) / tps) : 1;
    if (pl.n_split < 1) pl.n_split = 1;
  } else {
    pl.kernel = 0;
    pl.rows_per_cta = 16;
    const long total_max = prefix_max + B;
    const long base = (long)R * Hkv * ((M + pl.rows_per_cta - 1) / pl.rows_per_cta);
    const long target = 4L * num_sms;
    long ns = base > 0 ? (target + base - 1) / base : 1;
    const long max_split = (total_max + 255) / 256;
    if (ns > max_split) ns = max_split;
    if (ns < 1) ns = 1;
    long len = (total_max + ns - 1) / ns;
    len = (len + 63) / 64 * 64;
    ns = (total_max + len - 1) / len;
    pl.n_split = (int)ns;
    pl.split_len = (int)len;
  }
  if (pl.n_split > 1) {
    const size_t rows = (size_t)R * Hkv * pl.n_split * M;
    pl.ws_o_bytes = (rows * D * sizeof(float) + 255) / 256 * 256;
    pl.ws_lse_bytes = (rows * sizeof(float) + 255) / 256 * 256;
  }
  // tensor-core kernel: the work units in longest-first order, and per row
  // tile a count of finished splits (the last one merges the partials)
  if (pl.kernel == 1) {
    // order [R*n_split], n_valid [1], bad-request mask [ceil(R/32)]
    pl.ws_order_bytes =
        (((size_t)R * pl.n_split + 1 + (size_t)(R + 31) / 32) * sizeof(int32_t) + 255) / 256 * 256;
    // one CTA per work item when the prefix is split, else one per SM (at most
    // one per work item) walking the items
    const long n_items = (long)((M + 127) / 128) * Hkv * R * pl.n_split;
    pl.num_ctas = (int)(pl.n_split > 1 ? n_items : (n_items < num_sms ? n_items : num_sms));
    if (pl.n_split > 1)
      pl.ws_count_bytes =
          ((size_t)R * Hkv * ((M + 127) / 128) * sizeof(int32_t) + 255) / 256 * 256;
  }
  pl.workspace_bytes = pl.ws_o_bytes + pl.ws_lse_bytes + pl.ws_order_bytes + pl.ws_count_bytes;
  return pl;
}

cudaError_t launch_softmax(const SoftmaxParams& p, const SoftmaxPlan& plan, bool bf16,
                           cudaStream_t stream) {
  if (plan.kernel == 1) return launch_softmax_tc(p, plan, stream);
  return launch_softmax_simt(p, plan, bf16, stream);
}

}  // namespace flare

extern "C" {

const char* flare_status_string(flare_status s) {
  switch (s) {
    case FLARE_OK: return "FLARE_OK";
    case FLARE_ERR_INVALID_ARGUMENT: return "FLARE_ERR_INVALID_ARGUMENT";
    case FLARE_ERR_UNSUPPORTED: return "FLARE_ERR_UNSUPPORTED";
    case FLARE_ERR_CUDA: return "FLARE_ERR_CUDA";
    case FLARE_ERR_DEVICE_STATUS: return "FLARE_ERR_DEVICE_STATUS";
  }
  return "FLARE_ERR_UNKNOWN";
}

flare_status flare_block_linear_attn(const flare_linear_desc* d, const void* q, const void* k,
                                     const void* v, const float* log_decay, const float* beta,
                                     const float* state_pool, const int32_t* state_slot,
                                     void* out, int32_t* dev_status, void* stream) {
  flare_status st = check_linear(d);
  if (st != FLARE_OK) return st;
  if (!q || !k || !v || !log_decay || !beta || !state_pool || !state_slot || !out || !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(state_pool) ||
      !aligned16(out))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests == 0) return FLARE_OK;
  GdrParams p;
  memset(&p, 0, sizeof p);
  p.R = d->num_requests;
  p.B = d->block_len;
  p.Hk = d->num_qk_heads;
  p.Hv = d->num_v_heads;
  p.dk = d->head_dim_k;
  p.dv = d->head_dim_v;
  p.nslots = d->num_state_slots;
  p.scale = d->scale;
  p.q = q;
  p.k = k;
  p.v = v;
  p.log_decay = log_decay;
  p.beta = beta;
  p.state_pool = const_cast<float*>(state_pool);  // read only: write_state = 0
  p.state_slot = state_slot;
  p.out_blockend = out;
  p.write_state = 0;
  p.dev_status = dev_status;
  const bool bf16 = d->act_dtype == FLARE_DT_BF16;
  // bf16: the persistent tensor-core kernels for 128 x 128 states (B <= 32,
  // and 33..64 as one chunk), the one-CTA-per-item tensor-core kernel for the
  // other shapes; fp32 the CUDA-core recurrence
  cudaError_t e;
  if (bf16 && gdr_denoise_persist_supported(p.B, p.dk, p.dv))
    e = launch_gdr_denoise_persist(p, static_cast<cudaStream_t>(stream));
  else if (bf16 && gdr_denoise_chunk64_supported(p.B, p.dk, p.dv))
    e = launch_gdr_denoise_chunk64(p, static_cast<cudaStream_t>(stream));
  else if (bf16 && gdr_denoise_tc_supported(p.B, p.dk, p.dv))
    e = launch_gdr_denoise_tc(p, static_cast<cudaStream_t>(stream));
  else
    e = launch_gdr_recurrent(p, bf16, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_commit_state(const flare_linear_desc* d, const void* q, const void* k,
                                const void* v, const float* log_decay, const float* beta,
                                float* state_pool, const int32_t* state_slot,
                                const int32_t* accept_len, void* causal_out,
                                int32_t* dev_status, void* stream) {
  flare_status st = check_linear(d);
  if (st != FLARE_OK) return st;
  if (!k || !v || !log_decay || !beta || !state_pool || !state_slot || !accept_len ||
      !dev_status || (causal_out && !q))
    return FLARE_ERR_INVALID_ARGUMENT;
  if ((q && !aligned16(q)) || !aligned16(k) || !aligned16(v) || !aligned16(state_pool) ||
      (causal_out && !aligned16(causal_out)))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests == 0) return FLARE_OK;
  GdrParams p;
  memset(&p, 0, sizeof p);
  p.R = d->num_requests;
  p.B = d->block_len;
  p.Hk = d->num_qk_heads;
  p.Hv = d->num_v_heads;
  p.dk = d->head_dim_k;
  p.dv = d->head_dim_v;
  p.nslots = d->num_state_slots;
  p.scale = d->scale;
  p.q = causal_out ? q : nullptr;
  p.k = k;
  p.v = v;
  p.log_decay = log_decay;
  p.beta = beta;
  p.state_pool = state_pool;
  p.state_slot = state_slot;
  p.accept_len = accept_len;
  p.out_causal = causal_out;
  p.write_state = 1;
  p.dev_status = dev_status;
  const bool bf16 = d->act_dtype == FLARE_DT_BF16;
  // bf16 blocks of the 128 x 128 state without token-causal outputs take the
  // tensor-core chunkwise commit, the rest the register recurrence
  const cudaError_t e =
      (bf16 && !causal_out && gdr_commit_tc_supported(p.B, p.dk, p.dv))
          ? launch_gdr_commit_tc(p, static_cast<cudaStream_t>(stream))
          : launch_gdr_commit(p, bf16, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_verify_linear_attn(const flare_linear_desc* d, int32_t max_verify,
                                      const void* q, const void* k, const void* v,
                                      const float* log_decay, const float* beta,
                                      float* state_pool, const int32_t* state_slot,
                                      const int32_t* verify_len, void* out, float* verify_states,
                                      int32_t* dev_status, void* stream) {
  flare_status st = check_linear(d);
  if (st != FLARE_OK) return st;
  if (max_verify < 0) return FLARE_ERR_INVALID_ARGUMENT;
  if (!q || !k || !v || !log_decay || !beta || !state_pool || !state_slot || !verify_len ||
      !out || !dev_status || (max_verify > 0 && !verify_states))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(state_pool) ||
      !aligned16(out) || !aligned16(verify_states))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests == 0) return FLARE_OK;
  GdrParams p;
  memset(&p, 0, sizeof p);
  p.R = d->num_requests;
  p.B = d->block_len;
  p.Hk = d->num_qk_heads;
  p.Hv = d->num_v_heads;
  p.dk = d->head_dim_k;
  p.dv = d->head_dim_v;
  p.nslots = d->num_state_slots;
  p.scale = d->scale;
  p.q = q;
  p.k = k;
  p.v = v;
  p.log_decay = log_decay;
  p.beta = beta;
  p.state_pool = state_pool;
  p.state_slot = state_slot;
  p.out_causal = out;
  p.write_state = 1;
  p.verify_len = verify_len;
  p.max_verify = max_verify;
  p.verify_states = verify_states;
  p.dev_status = dev_status;
  const cudaError_t e = launch_gdr_verify(p, d->act_dtype == FLARE_DT_BF16,
                                          static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_verify_commit(const flare_linear_desc* d, int32_t max_verify,
                                 int32_t num_layers, const float* const* verify_states,
                                 float* const* state_pools, const int32_t* state_slot,
                                 const int32_t* accept, const int32_t* verify_len,
                                 int32_t* dev_status, void* stream) {
  flare_status st = check_linear(d);
  if (st != FLARE_OK) return st;
  if (max_verify < 0 || num_layers < 1) return FLARE_ERR_INVALID_ARGUMENT;
  if (num_layers > kMaxVerifyLayers) return FLARE_ERR_UNSUPPORTED;
  if (!verify_states || !state_pools || !state_slot || !accept || !verify_len || !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  VerifyCommitParams p;
  memset(&p, 0, sizeof p);
  for (int l = 0; l < num_layers; ++l) {
    if (!state_pools[l] || (max_verify > 0 && !verify_states[l]))
      return FLARE_ERR_INVALID_ARGUMENT;
    if (!aligned16(state_pools[l]) || !aligned16(verify_states[l]))
      return FLARE_ERR_INVALID_ARGUMENT;
    p.records[l] = verify_states[l];
    p.pools[l] = state_pools[l];
  }
  if (d->num_requests == 0 || max_verify == 0) return FLARE_OK;
  p.R = d->num_requests;
  p.max_verify = max_verify;
  p.nslots = d->num_state_slots;
  p.n_layers = num_layers;
  p.state_elems = (size_t)d->num_v_heads * d->head_dim_k * d->head_dim_v;
  p.state_slot = state_slot;
  p.accept = accept;
  p.verify_len = verify_len;
  p.dev_status = dev_status;
  const cudaError_t e = launch_verify_commit(p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_short_conv(const flare_conv_desc* d, const void* x, void* conv_state,
                              const int32_t* state_slot, const float* weight, const float* bias,
                              const int32_t* accept_len, void* out, int32_t* dev_status,
                              void* stream) {
  if (!d) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests < 0 || d->block_len < 1 || d->channels < 1 || d->num_state_slots < 1 ||
      d->width < 1 || !valid_dtype(d->act_dtype) ||
      (d->activation != FLARE_ACT_NONE && d->activation != FLARE_ACT_SILU))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->width > 4 || d->channels % 8 != 0) return FLARE_ERR_UNSUPPORTED;
  if (!x || !state_slot || !weight || !out || !dev_status || (d->width > 1 && !conv_state))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(x) || !aligned16(conv_state) || !aligned16(weight) || !aligned16(bias) ||
      !aligned16(out))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests == 0) return FLARE_OK;
  ConvParams p;
  memset(&p, 0, sizeof p);
  p.R = d->num_requests;
  p.B = d->block_len;
  p.C = d->channels;
  p.W = d->width;
  p.nslots = d->num_state_slots;
  p.silu = d->activation == FLARE_ACT_SILU;
  p.x = x;
  p.conv_state = conv_state;
  p.state_slot = state_slot;
  p.weight = weight;
  p.bias = bias;
  p.accept_len = accept_len;
  p.out = out;
  p.dev_status = dev_status;
  const cudaError_t e = launch_short_conv(p, d->act_dtype == FLARE_DT_BF16,
                                          static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_two_stream_fwd(const flare_two_stream_desc* d, const float* chunk_states,
                                  const void* k, const void* v, const float* log_decay,
                                  const float* beta, const void* q_noisy, const void* k_noisy,
                                  const void* v_noisy, const float* log_decay_noisy,
                                  const float* beta_noisy, void* out_noisy, int32_t* dev_status,
                                  void* stream) {
  if (!d) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_seqs < 0 || d->seq_len < 0 || d->chunk_len < 1 || d->block_len < 1 ||
      d->num_qk_heads < 1 || d->num_v_heads < 1 || d->num_v_heads % d->num_qk_heads != 0 ||
      !valid_dtype(d->act_dtype))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->chunk_len != two_stream_chunk_len() || d->seq_len % d->chunk_len != 0)
    return FLARE_ERR_UNSUPPORTED;
  const int B = d->block_len;
  if (B != 1 && B != 2 && B != 4 && B != 8 && B != 16) return FLARE_ERR_UNSUPPORTED;
  if (d->head_dim_k != 128 || d->head_dim_v != 128) return FLARE_ERR_UNSUPPORTED;
  if (!chunk_states || !k || !v || !log_decay || !beta || !q_noisy || !k_noisy || !v_noisy ||
      !log_decay_noisy || !beta_noisy || !out_noisy || !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(chunk_states) || !aligned16(k) || !aligned16(v) || !aligned16(q_noisy) ||
      !aligned16(k_noisy) || !aligned16(v_noisy) || !aligned16(out_noisy))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_seqs == 0 || d->seq_len == 0) return FLARE_OK;
  TwoStreamParams p;
  memset(&p, 0, sizeof p);
  p.N = d->num_seqs;
  p.L = d->seq_len;
  p.B = B;
  p.Hk = d->num_qk_heads;
  p.Hv = d->num_v_heads;
  p.dk = d->head_dim_k;
  p.dv = d->head_dim_v;
  p.scale = d->scale;
  p.chunk_states = chunk_states;
  p.k = k;
  p.v = v;
  p.g = log_decay;
  p.beta = beta;
  p.qn = q_noisy;
  p.kn = k_noisy;
  p.vn = v_noisy;
  p.gn = log_decay_noisy;
  p.betan = beta_noisy;
  p.out = out_noisy;
  p.dev_status = dev_status;
  const cudaError_t e = launch_two_stream_fwd(p, d->act_dtype == FLARE_DT_BF16,
                                              static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_softmax_workspace_size(const flare_softmax_desc* d, size_t* bytes) {
  flare_status st = check_softmax(d);
  if (st != FLARE_OK) return st;
  if (!bytes) return FLARE_ERR_INVALID_ARGUMENT;
  *bytes = d->num_requests == 0 ? 0 : plan_for(d).workspace_bytes;
  return FLARE_OK;
}

flare_status flare_block_softmax_attn(const flare_softmax_desc* d, const void* q,
                                      const void* k_blk, const void* v_blk, const void* k_pool,
                                      const void* v_pool, const int32_t* page_table,
                                      const int32_t* prefix_len, void* out, float* lse,
                                      void* workspace, size_t workspace_bytes,
                                      int32_t* dev_status, void* stream) {
  flare_status st = check_softmax(d);
  if (st != FLARE_OK) return st;
  if (!q || !k_blk || !v_blk || !prefix_len || !out || !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->max_pages_per_req > 0 && (!k_pool || !v_pool || !page_table))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(q) || !aligned16(k_blk) || !aligned16(v_blk) || !aligned16(k_pool) ||
      !aligned16(v_pool) || !aligned16(out))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests == 0) return FLARE_OK;
  const SoftmaxPlan plan = plan_for(d);
  if (workspace_bytes < plan.workspace_bytes) return FLARE_ERR_INVALID_ARGUMENT;
  if (plan.workspace_bytes && (!workspace || ((uintptr_t)workspace & 255u)))
    return FLARE_ERR_INVALID_ARGUMENT;
  SoftmaxParams p = softmax_params(d);
  p.q = q;
  p.k_blk = k_blk;
  p.v_blk = v_blk;
  p.k_pool = k_pool;
  p.v_pool = v_pool;
  p.page_table = page_table;
  p.prefix_len = prefix_len;
  p.out = out;
  p.lse = lse;
  p.n_split = plan.n_split;
  p.split_len = plan.split_len;
  if (plan.workspace_bytes) {
    char* ws = static_cast<char*>(workspace);
    if (plan.ws_o_bytes) {
      p.ws_o = reinterpret_cast<float*>(ws);
      p.ws_lse = reinterpret_cast<float*>(ws + plan.ws_o_bytes);
    }
    if (plan.ws_order_bytes) {
      p.order = reinterpret_cast<int32_t*>(ws + plan.ws_o_bytes + plan.ws_lse_bytes);
      p.n_valid = p.order + (size_t)p.R * plan.n_split;
      p.bad_mask = reinterpret_cast<uint32_t*>(p.n_valid + 1);
    }
    if (plan.ws_count_bytes)
      p.counters = reinterpret_cast<int32_t*>(ws + plan.ws_o_bytes + plan.ws_lse_bytes +
                                              plan.ws_order_bytes);
  }
  p.dev_status = dev_status;
  const cudaError_t e = launch_softmax(p, plan, d->act_dtype == FLARE_DT_BF16,
                                       static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_append_kv(const flare_softmax_desc* d, const void* k_blk, const void* v_blk,
                             void* k_pool, void* v_pool, const int32_t* page_table,
                             const int32_t* prefix_len, const int32_t* append_len,
                             int32_t* dev_status, void* stream) {
  flare_status st = check_softmax(d);
  if (st != FLARE_OK) return st;
  if (!k_blk || !v_blk || !k_pool || !v_pool || !page_table || !prefix_len || !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(k_blk) || !aligned16(v_blk) || !aligned16(k_pool) || !aligned16(v_pool))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests == 0) return FLARE_OK;
  SoftmaxParams p = softmax_params(d);
  p.k_blk = k_blk;
  p.v_blk = v_blk;
  p.page_table = page_table;
  p.prefix_len = prefix_len;
  p.dev_status = dev_status;
  const int elem = d->act_dtype == FLARE_DT_BF16 ? 2 : 4;
  const cudaError_t e = launch_append_kv(p, append_len, k_pool, v_pool, elem,
                                         static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_tree_softmax_workspace_size(const flare_softmax_desc* d, size_t* bytes) {
  flare_status st = check_tree_softmax(d);
  if (st != FLARE_OK) return st;
  if (!bytes) return FLARE_ERR_INVALID_ARGUMENT;
  *bytes = d->num_requests == 0 ? 0 : tree_plan_for(d).workspace_bytes;
  return FLARE_OK;
}

flare_status flare_tree_softmax_attn(const flare_softmax_desc* d, const void* q,
                                     const void* k_blk, const void* v_blk, const void* k_pool,
                                     const void* v_pool, const int32_t* page_table,
                                     const int32_t* prefix_len, const int32_t* parent,
                                     const int32_t* node_len, void* out, float* lse,
                                     void* workspace, size_t workspace_bytes,
                                     int32_t* dev_status, void* stream) {
  flare_status st = check_tree_softmax(d);
  if (st != FLARE_OK) return st;
  if (!q || !k_blk || !v_blk || !prefix_len || !parent || !node_len || !out || !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->max_pages_per_req > 0 && (!k_pool || !v_pool || !page_table))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(q) || !aligned16(k_blk) || !aligned16(v_blk) || !aligned16(k_pool) ||
      !aligned16(v_pool) || !aligned16(out))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests == 0) return FLARE_OK;
  const TreeSoftmaxPlan plan = tree_plan_for(d);
  if (workspace_bytes < plan.workspace_bytes || !workspace || ((uintptr_t)workspace & 255u))
    return FLARE_ERR_INVALID_ARGUMENT;
  TreeSoftmaxParams p;
  memset(&p, 0, sizeof p);
  p.R = d->num_requests;
  p.N = d->block_len;
  p.Hq = d->num_q_heads;
  p.Hkv = d->num_kv_heads;
  p.G = d->num_q_heads / d->num_kv_heads;
  p.D = d->head_dim;
  p.page_size = d->page_size;
  p.num_pages = d->num_pages;
  p.max_pages = d->max_pages_per_req;
  p.scale_log2 = d->scale * 1.4426950408889634f;
  p.q = q;
  p.k_blk = k_blk;
  p.v_blk = v_blk;
  p.k_pool = k_pool;
  p.v_pool = v_pool;
  p.page_table = page_table;
  p.prefix_len = prefix_len;
  p.parent = parent;
  p.node_len = node_len;
  p.out = out;
  p.lse = lse;
  p.gangs = plan.gangs;
  p.row_tiles = plan.row_tiles;
  p.tile_base = plan.tile_base;
  p.tile_rows = plan.tile_rows;
  char* ws = static_cast<char*>(workspace);
  p.bad = reinterpret_cast<int32_t*>(ws + plan.bad_off);
  p.n_cuts = reinterpret_cast<int32_t*>(ws + plan.n_cuts_off);
  p.cuts = ws + plan.cuts_off;
  p.counts = reinterpret_cast<int32_t*>(ws + plan.counts_off);
  p.n_counts = plan.n_counts;
  p.join = plan.join;
  p.anc = reinterpret_cast<uint64_t*>(ws + plan.anc_off);
  p.part_o = reinterpret_cast<float*>(ws + plan.part_o_off);
  p.part_lse = reinterpret_cast<float*>(ws + plan.part_lse_off);
  p.dev_status = dev_status;
  const cudaError_t e = launch_tree_softmax(p, d->act_dtype == FLARE_DT_BF16,
                                            static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_tree_linear_attn(const flare_linear_desc* d, const void* q, const void* k,
                                    const void* v, const float* log_decay, const float* beta,
                                    const float* state_pool, const int32_t* state_slot,
                                    const int32_t* parent, const int32_t* node_len, void* out,
                                    int32_t* dev_status, void* stream) {
  flare_status st = check_linear(d);
  if (st != FLARE_OK) return st;
  if (!q || !k || !v || !log_decay || !beta || !state_pool || !state_slot || !parent ||
      !node_len || !out || !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(state_pool) ||
      !aligned16(out))
    return FLARE_ERR_INVALID_ARGUMENT;
  if ((int64_t)d->num_requests * d->num_v_heads > INT32_MAX) return FLARE_ERR_UNSUPPORTED;
  if (d->num_requests == 0) return FLARE_OK;
  GdrParams p;
  memset(&p, 0, sizeof p);
  p.R = d->num_requests;
  p.B = d->block_len;
  p.Hk = d->num_qk_heads;
  p.Hv = d->num_v_heads;
  p.dk = d->head_dim_k;
  p.dv = d->head_dim_v;
  p.nslots = d->num_state_slots;
  p.scale = d->scale;
  p.q = q;
  p.k = k;
  p.v = v;
  p.log_decay = log_decay;
  p.beta = beta;
  p.state_pool = const_cast<float*>(state_pool);  // read only
  p.state_slot = state_slot;
  p.parent = parent;
  p.node_len = node_len;
  p.out_causal = out;
  p.dev_status = dev_status;
  const cudaError_t e = launch_tree_linear(p, d->act_dtype == FLARE_DT_BF16,
                                           static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_tree_verify_workspace_size(const flare_tree_verify_desc* d, size_t* bytes) {
  flare_status st = check_tree_verify(d);
  if (st != FLARE_OK) return st;
  if (!bytes) return FLARE_ERR_INVALID_ARGUMENT;
  int chunk, n_chunks;
  *bytes = tree_verify_workspace(d, &chunk, &n_chunks);
  return FLARE_OK;
}

flare_status flare_tree_verify(const flare_tree_verify_desc* d, const void* logits,
                               const float* draft_probs, const int32_t* token,
                               const int32_t* parent, const int32_t* node_len,
                               const float* uniform, const float* noise, int32_t* path,
                               int32_t* path_len, int32_t* next_token, float* node_logp,
                               void* workspace, size_t workspace_bytes, int32_t* dev_status,
                               void* stream) {
  flare_status st = check_tree_verify(d);
  if (st != FLARE_OK) return st;
  const bool sample = d->mode == FLARE_VERIFY_SAMPLE;
  if (!logits || !token || !parent || !node_len || !path || !path_len || !next_token ||
      !node_logp || !dev_status || (sample && (!uniform || !noise)))
    return FLARE_ERR_INVALID_ARGUMENT;
  const size_t elem = d->logits_dtype == FLARE_DT_BF16 ? 2 : 4;
  if ((uintptr_t)logits % elem || (uintptr_t)draft_probs % 4 || (uintptr_t)noise % 4)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests == 0) return FLARE_OK;
  TreeVerifyParams p;
  memset(&p, 0, sizeof p);
  const size_t need = tree_verify_workspace(d, &p.chunk, &p.n_chunks);
  if (workspace_bytes < need || !workspace || ((uintptr_t)workspace & 255u))
    return FLARE_ERR_INVALID_ARGUMENT;
  p.R = d->num_requests;
  p.N = d->num_nodes;
  p.V = d->vocab_size;
  p.greedy = !sample;
  p.inv_temp = sample ? d->inv_temperature : 1.f;
  p.logits = logits;
  p.draft_probs = draft_probs;
  p.token = token;
  p.parent = parent;
  p.node_len = node_len;
  p.uniform = uniform;
  p.noise = noise;
  p.path = path;
  p.path_len = path_len;
  p.next_token = next_token;
  p.node_logp = node_logp;
  p.stats = static_cast<float4*>(workspace);
  p.dev_status = dev_status;
  const cudaError_t e = launch_tree_verify(p, d->logits_dtype == FLARE_DT_BF16,
                                           static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_tree_commit_state(const flare_linear_desc* d, const void* k, const void* v,
                                     const float* log_decay, const float* beta,
                                     float* state_pool, const int32_t* src_slot,
                                     const int32_t* dst_slot, const int32_t* path,
                                     const int32_t* path_len, int32_t* dev_status, void* stream) {
  flare_status st = check_linear(d);
  if (st != FLARE_OK) return st;
  if (!k || !v || !log_decay || !beta || !state_pool || !src_slot || !dst_slot || !path ||
      !path_len || !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(k) || !aligned16(v) || !aligned16(state_pool)) return FLARE_ERR_INVALID_ARGUMENT;
  if ((int64_t)d->num_requests * d->num_v_heads > INT32_MAX) return FLARE_ERR_UNSUPPORTED;
  if (d->num_requests == 0) return FLARE_OK;
  GdrParams p;
  memset(&p, 0, sizeof p);
  p.R = d->num_requests;
  p.B = d->block_len;
  p.Hk = d->num_qk_heads;
  p.Hv = d->num_v_heads;
  p.dk = d->head_dim_k;
  p.dv = d->head_dim_v;
  p.nslots = d->num_state_slots;
  p.k = k;
  p.v = v;
  p.log_decay = log_decay;
  p.beta = beta;
  p.state_pool = state_pool;
  p.state_slot = src_slot;
  p.dst_slot = dst_slot;
  p.accept_len = path_len;
  p.path = path;
  p.write_state = 1;
  p.dev_status = dev_status;
  const cudaError_t e = launch_tree_commit(p, d->act_dtype == FLARE_DT_BF16,
                                           static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_tree_append_kv(const flare_softmax_desc* d, int32_t num_layers,
                                  const void* const* k_blk, const void* const* v_blk,
                                  void* const* k_pool, void* const* v_pool,
                                  const int32_t* page_table, const int32_t* prefix_len,
                                  const int32_t* path, const int32_t* path_len,
                                  int32_t* dev_status, void* stream) {
  flare_status st = check_tree_softmax(d);
  if (st != FLARE_OK) return st;
  if (num_layers < 1) return FLARE_ERR_INVALID_ARGUMENT;
  if (num_layers > kMaxAppendLayers) return FLARE_ERR_UNSUPPORTED;
  if (!k_blk || !v_blk || !k_pool || !v_pool || !page_table || !prefix_len || !path ||
      !path_len || !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  TreeAppendParams p;
  memset(&p, 0, sizeof p);
  for (int l = 0; l < num_layers; ++l) {
    if (!k_blk[l] || !v_blk[l] || !k_pool[l] || !v_pool[l] || !aligned16(k_blk[l]) ||
        !aligned16(v_blk[l]) || !aligned16(k_pool[l]) || !aligned16(v_pool[l]))
      return FLARE_ERR_INVALID_ARGUMENT;
    p.k_blk[l] = k_blk[l];
    p.v_blk[l] = v_blk[l];
    p.k_pool[l] = k_pool[l];
    p.v_pool[l] = v_pool[l];
  }
  if (d->num_requests == 0) return FLARE_OK;
  p.R = d->num_requests;
  p.N = d->block_len;
  p.Hkv = d->num_kv_heads;
  p.D = d->head_dim;
  p.page_size = d->page_size;
  p.num_pages = d->num_pages;
  p.max_pages = d->max_pages_per_req;
  p.n_layers = num_layers;
  p.elem_bytes = d->act_dtype == FLARE_DT_BF16 ? 2 : 4;
  p.page_table = page_table;
  p.prefix_len = prefix_len;
  p.path = path;
  p.path_len = path_len;
  p.dev_status = dev_status;
  const cudaError_t e = launch_tree_append(p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_rotary_table(const flare_rotary_freq_desc* d, uint64_t* table, void* stream) {
  if (!d || !table || !aligned(table, 8)) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->scaling != FLARE_ROTARY_PLAIN && d->scaling != FLARE_ROTARY_LINEAR &&
      d->scaling != FLARE_ROTARY_BASE && d->scaling != FLARE_ROTARY_BY_PARTS)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!(d->base >= 1.0 && d->base < 1e300) ||
      (d->scaling != FLARE_ROTARY_PLAIN && !(d->factor > 0.0 && d->factor < 1e100)))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->scaling == FLARE_ROTARY_BY_PARTS &&
      !(d->original_len > 0.0 && d->original_len < 1e100 && d->low_turns >= 0.0 &&
        d->low_turns < d->high_turns && d->high_turns < 1e100))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->rotary_dim < 16 || d->rotary_dim > 256 || d->rotary_dim % 16) return FLARE_ERR_UNSUPPORTED;
  const cudaError_t e = launch_rotary_table(*d, table, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_rotary(const flare_rotary_desc* d, const void* q, const void* k,
                          const uint64_t* table, const int32_t* position,
                          const int32_t* prefix_len, const int32_t* token_len,
                          const int32_t* parent, const int32_t* token_start, void* q_out,
                          void* k_out, int32_t* dev_status, void* stream) {
  flare_status st = check_rotary(d, token_start != nullptr, false);
  if (st != FLARE_OK || no_rows(d, token_start != nullptr)) return st;
  if ((!q && !k) || !q != !q_out || !k != !k_out || !table || !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (token_start && (token_len || parent)) return FLARE_ERR_INVALID_ARGUMENT;
  if (parent && d->block_len > kMaxTreeNodes) return FLARE_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) ||
      !aligned(table, 8))
    return FLARE_ERR_INVALID_ARGUMENT;
  return rotary(d, q, k, nullptr, table, position, prefix_len, token_len, parent, token_start,
                nullptr, q_out, k_out, nullptr, nullptr, dev_status, stream);
}

flare_status flare_rotary_append_kv(const flare_rotary_desc* d, const void* q, const void* k,
                                    const void* v, const uint64_t* table,
                                    const int32_t* position, const int32_t* prefix_len,
                                    const int32_t* token_len, const int32_t* token_start,
                                    const int32_t* page_table, void* q_out, void* k_out,
                                    void* k_pool, void* v_pool, int32_t* dev_status,
                                    void* stream) {
  flare_status st = check_rotary(d, token_start != nullptr, true);
  if (st != FLARE_OK || no_rows(d, token_start != nullptr)) return st;
  if (!k || !v || !q != !q_out || !table || !prefix_len || !page_table || !k_pool || !v_pool ||
      !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (token_start && token_len) return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_out) ||
      !aligned16(k_pool) || !aligned16(v_pool) || !aligned(table, 8))
    return FLARE_ERR_INVALID_ARGUMENT;
  return rotary(d, q, k, v, table, position, prefix_len, token_len, nullptr, token_start,
                page_table, q_out, k_out, k_pool, v_pool, dev_status, stream);
}

flare_status flare_tree_logits(const flare_tree_logits_desc* d, const void* logits,
                               const int32_t* history, const int32_t* history_len,
                               const int32_t* output_start, const int32_t* token,
                               const int32_t* parent, const int32_t* node_len,
                               const float* repetition, const float* presence,
                               const float* frequency, const int32_t* bias_token,
                               const float* bias_value, const int32_t* bias_len,
                               const uint32_t* mask, void* out, int32_t* dev_status,
                               void* stream) {
  if (!d) return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_requests < 0 || d->num_nodes < 1 || d->vocab_size < 1 || d->max_history < 0 ||
      d->max_bias < 0 || !valid_dtype(d->logits_dtype))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (d->num_nodes > kMaxTreeNodes || d->vocab_size > (1 << 24) || d->max_history > (1 << 24) ||
      d->max_bias > 65536)
    return FLARE_ERR_UNSUPPORTED;
  if (d->num_requests == 0) return FLARE_OK;
  if (!logits || !out || !dev_status || (history && !history_len) ||
      (token && (!parent || !node_len)) || !bias_token != !bias_value || !bias_token != !bias_len)
    return FLARE_ERR_INVALID_ARGUMENT;
  const size_t e = elem_bytes(d->logits_dtype);
  const size_t bytes = (size_t)d->num_requests * d->num_nodes * d->vocab_size * e;
  if (!aligned(logits, e) || !aligned(out, e) ||
      (out != logits && overlap(logits, bytes, out, bytes)) ||
      !aligned4({history, history_len, output_start, token, parent, node_len, repetition, presence,
                 frequency, bias_token, bias_value, bias_len, mask, dev_status}))
    return FLARE_ERR_INVALID_ARGUMENT;
  TreeLogitsParams p;
  memset(&p, 0, sizeof p);
  p.R = d->num_requests;
  p.N = d->num_nodes;
  p.V = d->vocab_size;
  p.H = d->max_history;
  p.max_bias = d->max_bias;
  p.logits = logits;
  p.history = history;
  p.history_len = history_len;
  p.output_start = output_start;
  p.token = token;
  p.parent = parent;
  p.node_len = node_len;
  p.repetition = repetition;
  p.presence = presence;
  p.frequency = frequency;
  p.bias_token = bias_token;
  p.bias_value = bias_value;
  p.bias_len = bias_len;
  p.mask = mask;
  p.out = out;
  p.dev_status = dev_status;
  const cudaError_t err = launch_tree_logits(p, d->logits_dtype == FLARE_DT_BF16, device_sms(),
                                             static_cast<cudaStream_t>(stream));
  return err == cudaSuccess ? FLARE_OK
                            : err == cudaErrorInvalidConfiguration ? FLARE_ERR_UNSUPPORTED
                                                                   : FLARE_ERR_CUDA;
}

flare_status flare_block_norm(const flare_block_norm_desc* d, const void* x, const void* gate,
                              const void* residual, const float* post_weight,
                              const float* pre_weight, void* y, void* h, void* stream) {
  flare_status st = check_block_norm(d);
  if (st != FLARE_OK || d->num_tokens == 0) return st;
  if (!x || (!y && !h) || !h != !d->pre_norm) return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(x) || !aligned16(gate) || !aligned16(residual) || !aligned16(post_weight) ||
      !aligned16(pre_weight) || !aligned16(y) || !aligned16(h))
    return FLARE_ERR_INVALID_ARGUMENT;
  BlockNormParams p = block_norm_params(d, x, gate, residual, post_weight, pre_weight);
  const Rows in[3] = {{x, p.x_stride, p.W}, {gate, p.gate_stride, p.W}, {residual, p.W, p.W}};
  const Rows out[2] = {{y, p.W, p.W}, {h, p.W, p.W}};
  if (!outputs_clear(in, 3, out, 2, false, p.T, elem_bytes(d->act_dtype)))
    return FLARE_ERR_INVALID_ARGUMENT;
  p.y = y;
  p.h = h;
  const cudaError_t e = launch_block_norm(p, d->act_dtype == FLARE_DT_BF16, device_sms(),
                                          static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_block_norm_bwd_workspace_size(const flare_block_norm_desc* d, size_t* bytes) {
  flare_status st = check_block_norm(d);
  if (st != FLARE_OK) return st;
  if (!bytes) return FLARE_ERR_INVALID_ARGUMENT;
  *bytes = (size_t)block_norm_bwd_ctas(d->num_tokens, d->width, d->pre_norm,
                                       d->act_dtype == FLARE_DT_BF16, device_sms()) * 2 * d->width * sizeof(float);
  return FLARE_OK;
}

flare_status flare_block_norm_bwd(const flare_block_norm_desc* d, const void* x,
                                  const void* gate, const void* residual,
                                  const float* post_weight, const float* pre_weight,
                                  const void* dy, const void* dh, void* dx, void* dgate,
                                  void* dresidual, float* dpost_weight, float* dpre_weight,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  flare_status st = check_block_norm(d);
  if (st != FLARE_OK) return st;
  if ((dpost_weight && !d->post_norm) || (dpre_weight && !d->pre_norm) ||
      (d->num_tokens > 0 &&
       (!x || !dx || !gate != !dgate || (dresidual && !residual) || !dh != !d->pre_norm ||
        (!dy && !dh))))
    return FLARE_ERR_INVALID_ARGUMENT;
  if (!aligned16(x) || !aligned16(gate) || !aligned16(residual) || !aligned16(post_weight) ||
      !aligned16(pre_weight) || !aligned16(dy) || !aligned16(dh) || !aligned16(dx) ||
      !aligned16(dgate) || !aligned16(dresidual) || !aligned(dpost_weight, 4) ||
      !aligned(dpre_weight, 4))
    return FLARE_ERR_INVALID_ARGUMENT;
  BlockNormParams p = block_norm_params(d, x, gate, residual, post_weight, pre_weight);
  const Rows in[5] = {{x, p.x_stride, p.W}, {gate, p.gate_stride, p.W}, {residual, p.W, p.W},
                      {dy, p.W, p.W}, {dh, p.W, p.W}};
  const Rows out[3] = {{dx, p.x_stride, p.W}, {dgate, p.gate_stride, p.W}, {dresidual, p.W, p.W}};
  if (!outputs_clear(in, 5, out, 3, false, p.T, elem_bytes(d->act_dtype)))
    return FLARE_ERR_INVALID_ARGUMENT;
  const bool weights = dpost_weight || dpre_weight;
  if (weights) {
    size_t need;
    flare_block_norm_bwd_workspace_size(d, &need);
    if (workspace_bytes < need || (need && !workspace) || !aligned(workspace, 256))
      return FLARE_ERR_INVALID_ARGUMENT;
  }
  p.dy = dy;
  p.dh = dh;
  p.dx = dx;
  p.dgate = dgate;
  p.dres = dresidual;
  p.dwpost = dpost_weight;
  p.dwpre = dpre_weight;
  p.part = weights ? static_cast<float*>(workspace) : nullptr;
  const cudaError_t e = launch_block_norm_bwd(p, d->act_dtype == FLARE_DT_BF16, device_sms(),
                                              static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_debug_gather_prefix(const flare_softmax_desc* d, const void* k_pool,
                                       const void* v_pool, const int32_t* page_table,
                                       const int32_t* prefix_len, int32_t request, void* k_out,
                                       void* v_out, int32_t* dev_status, void* stream) {
  flare_status st = check_softmax(d);
  if (st != FLARE_OK) return st;
  if (!k_pool || !v_pool || !page_table || !prefix_len || !k_out || !v_out || !dev_status)
    return FLARE_ERR_INVALID_ARGUMENT;
  if (request < 0 || request >= d->num_requests) return FLARE_ERR_INVALID_ARGUMENT;
  SoftmaxParams p = softmax_params(d);
  p.k_pool = k_pool;
  p.v_pool = v_pool;
  p.page_table = page_table;
  p.prefix_len = prefix_len;
  p.dev_status = dev_status;
  const cudaError_t e = launch_gather_prefix(p, request, k_out, v_out,
                                             d->act_dtype == FLARE_DT_BF16,
                                             static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

flare_status flare_debug_wait_timeout(int32_t* dev_status, uint64_t limit_ns, void* stream) {
  if (!dev_status || limit_ns < 1000ull || limit_ns > 1000000000ull)
    return FLARE_ERR_INVALID_ARGUMENT;
  const cudaError_t e =
      launch_debug_wait_timeout(dev_status, limit_ns, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FLARE_OK : FLARE_ERR_CUDA;
}

uint64_t flare_launch_count(void) { return g_launches.load(std::memory_order_relaxed); }

flare_status flare_read_status(const int32_t* dev_status, void* stream, int32_t* bits_out) {
  if (!dev_status) return FLARE_ERR_INVALID_ARGUMENT;
  int32_t bits = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (cudaMemcpyAsync(&bits, dev_status, sizeof bits, cudaMemcpyDeviceToHost, s) != cudaSuccess)
    return FLARE_ERR_CUDA;
  if (cudaStreamSynchronize(s) != cudaSuccess) return FLARE_ERR_CUDA;
  if (bits_out) *bits_out = bits;
  return bits ? FLARE_ERR_DEVICE_STATUS : FLARE_OK;
}

}  // extern "C"
