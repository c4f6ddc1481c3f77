// Internal launch interface between the C ABI layer and the kernels.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace flare {

constexpr int kNumSMs = 152;  // GB300: 2 dies x 76 SMs (re-read at run time)

// Counts kernel launches for flare_launch_count().
void note_launches(int n);

struct GdrParams {
  int R, B, Hk, Hv, dk, dv, nslots;
  float scale;
  const void* q;  // [R,B,Hk,dk], nullable when no readout is asked
  const void* k;  // [R,B,Hk,dk]
  const void* v;  // [R,B,Hv,dv]
  const float* log_decay;  // [R,B,Hv]
  const float* beta;       // [R,B,Hv]
  float* state_pool;       // [nslots,Hv,dk,dv]; written only when write_state
  const int32_t* state_slot;  // [R]
  const int32_t* accept_len;  // [R] or nullptr (= B)
  void* out_blockend;         // [R,B,Hv,dv] or nullptr
  void* out_causal;           // [R,B,Hv,dv] or nullptr
  int write_state;
  // AR-Trust verify round
  const int32_t* verify_len;  // [R] or nullptr
  int max_verify;
  float* verify_states;       // [R,max_verify,Hv,dk,dv]
  // drafted trees (B = nodes per tree)
  const int32_t* parent;      // [R,B]
  const int32_t* node_len;    // [R]
  const int32_t* path;        // [R,B] accepted nodes: commit along a path
  const int32_t* dst_slot;    // [R] where that commit writes
  int32_t* dev_status;
};

struct SoftmaxParams {
  int R, B, Hq, Hkv, G, D, page_size, num_pages, max_pages;
  float scale_log2;  // logit scale * log2(e)
  int causal;
  const uint8_t* row_type;  // per-row types (0 = token-causal) or nullptr
  int row_type_stride;      // 0 (one layout for the batch) or B (per request)
  const void* q;      // [R,B,Hq,D]
  const void* k_blk;  // [R,B,Hkv,D]
  const void* v_blk;
  const void* k_pool;  // [num_pages,Hkv,page_size,D]
  const void* v_pool;
  const int32_t* page_table;  // [R,max_pages]
  const int32_t* prefix_len;  // [R]
  void* out;                  // [R,B,Hq,D]
  float* lse;                 // [R,B,Hq] or nullptr
  float* ws_o;                // split partial outputs [R*Hkv][n_split][B*G][D]
  float* ws_lse;              // split partial lse     [R*Hkv][n_split][B*G]
  int n_split, split_len;
  int32_t* order;             // [R*n_split] valid work units (r, split), longest first
  int32_t* n_valid;           // number of valid work units in `order`
  uint32_t* bad_mask;         // [ceil(R/32)] requests with a bad prefix length or page id
  int32_t* counters;          // [R*Hkv*ceil(B*G/128)] finished splits per row tile (n_split > 1)
  int32_t* dev_status;
};

// Work decomposition of the softmax call; identical for the workspace query
// and the launch.
struct SoftmaxPlan {
  int kernel;  // 0 = CUDA-core kernel, 1 = tensor-core kernel
  int rows_per_cta;
  int n_split;
  int split_len;
  int num_ctas;  // tensor-core kernel: CTAs launched
  size_t ws_o_bytes, ws_lse_bytes, ws_order_bytes, ws_count_bytes;
  size_t workspace_bytes;
};

size_t gdr_recurrent_smem_bytes(int dk, int dv, int threads);
bool gdr_denoise_tc_supported(int B, int dk, int dv);
bool gdr_denoise_persist_supported(int B, int dk, int dv);
cudaError_t launch_gdr_denoise_persist(const GdrParams& p, cudaStream_t stream);
bool gdr_denoise_chunk64_supported(int B, int dk, int dv);
cudaError_t launch_gdr_denoise_chunk64(const GdrParams& p, cudaStream_t stream);
cudaError_t launch_gdr_commit(const GdrParams& p, bool bf16, cudaStream_t stream);
bool gdr_commit_tc_supported(int B, int dk, int dv);
cudaError_t launch_gdr_commit_tc(const GdrParams& p, cudaStream_t stream);
cudaError_t launch_gdr_verify(const GdrParams& p, bool bf16, cudaStream_t stream);

constexpr int kMaxVerifyLayers = 64;
struct VerifyCommitParams {
  int R, max_verify, nslots, n_layers;
  size_t state_elems;  // Hv * dk * dv
  const float* records[kMaxVerifyLayers];
  float* pools[kMaxVerifyLayers];
  const int32_t* state_slot;
  const int32_t* accept;
  const int32_t* verify_len;
  int32_t* dev_status;
};
cudaError_t launch_verify_commit(const VerifyCommitParams& p, cudaStream_t stream);

struct ConvParams {
  int R, B, C, W, nslots, silu;
  const void* x;              // [R,B,C]
  void* conv_state;           // [nslots,W-1,C]
  const int32_t* state_slot;  // [R]
  const float* weight;        // [C,W]
  const float* bias;          // [C] or nullptr
  const int32_t* accept_len;  // [R] or nullptr (no commit)
  void* out;                  // [R,B,C]
  int32_t* dev_status;
};
cudaError_t launch_short_conv(const ConvParams& p, bool bf16, cudaStream_t stream);

struct TwoStreamParams {
  int N, L, B, Hk, Hv, dk, dv;
  float scale;
  const float* chunk_states;  // [N,Hv,L/64,dk,dv]
  const void* k;              // clean [N,L,Hk,dk]
  const void* v;              // clean [N,L,Hv,dv]
  const float* g;             // clean log-gates [N,L,Hv]
  const float* beta;
  const void* qn;             // noisy [N,L,Hk,dk]
  const void* kn;
  const void* vn;             // noisy [N,L,Hv,dv]
  const float* gn;
  const float* betan;
  void* out;                  // [N,L,Hv,dv]
  int32_t* dev_status;
};
int two_stream_chunk_len();
cudaError_t launch_two_stream_fwd(const TwoStreamParams& p, bool bf16, cudaStream_t stream);
bool two_stream_chunk_supported(int B, int dk, int dv);
cudaError_t launch_two_stream_chunk(const TwoStreamParams& p, cudaStream_t stream);
cudaError_t launch_gdr_denoise_tc(const GdrParams& p, cudaStream_t stream);
cudaError_t launch_gdr_recurrent(const GdrParams& p, bool bf16, cudaStream_t stream);

// Softmax attention of drafted trees.  Work is cut by key tiles (tree_sched.cuh):
// `gangs` spans of the batch's tiles, each walked by `row_tiles` CTAs.
struct TreeSoftmaxParams {
  int R, N, Hq, Hkv, G, D, page_size, num_pages, max_pages;
  float scale_log2;           // logit scale * log2(e)
  const void* q;              // [R,N,Hq,D]
  const void* k_blk;          // [R,N,Hkv,D]
  const void* v_blk;
  const void* k_pool;         // [num_pages,Hkv,page_size,D]
  const void* v_pool;
  const int32_t* page_table;  // [R,max_pages]
  const int32_t* prefix_len;  // [R]
  const int32_t* parent;      // [R,N]
  const int32_t* node_len;    // [R]
  void* out;                  // [R,N,Hq,D]
  float* lse;                 // [R,N,Hq] or nullptr
  int gangs, row_tiles;       // row_tiles: CTAs per gang
  int tile_base, tile_rows;   // query rows of a row tile, and of a CTA's one or two
  int32_t* bad;               // [R] whether a request is skipped
  int32_t* n_cuts;
  void* cuts;                 // [n_cuts <= gangs] TreeCut: items for tree_finish_kernel to merge
  int join;                   // pieces of an item that its last one merges itself
  int n_counts;
  int32_t* counts;            // [gangs,row_tiles,1 or 2] stored pieces of the item a gang starts
  uint64_t* anc;              // [R,N] path of each node as a bit set
  float* part_o;              // [2 gangs row_tiles][tile_rows][D] partial outputs
  float* part_lse;            // [2 gangs row_tiles][tile_rows]
  int32_t* dev_status;
};

struct TreeSoftmaxPlan {
  int gangs, row_tiles, tile_base, tile_rows, n_counts, join;
  size_t bad_off, n_cuts_off, cuts_off, counts_off, anc_off, part_o_off, part_lse_off, workspace_bytes;
};

TreeSoftmaxPlan plan_tree_softmax(int R, int N, int Hq, int Hkv, int D, int page_size,
                                  int max_pages, bool bf16, int num_sms);
cudaError_t launch_tree_softmax(const TreeSoftmaxParams& p, bool bf16, cudaStream_t stream);
// The bf16 attention's tensor maps (queries, nodes' keys and values, pools).
struct TreeSoftmaxTc {
  CUtensorMap q, kblk, vblk, kpool, vpool;
};
cudaError_t prepare_tree_softmax_tc(const TreeSoftmaxParams& p, TreeSoftmaxTc* tc);
cudaError_t launch_tree_softmax_tc(const TreeSoftmaxParams& p, const TreeSoftmaxTc& tc,
                                   cudaStream_t stream);

cudaError_t launch_tree_linear(const GdrParams& p, bool bf16, cudaStream_t stream);
bool tree_linear_tc_supported(int dk, int dv);
cudaError_t launch_tree_linear_tc(const GdrParams& p, cudaStream_t stream);
cudaError_t launch_tree_commit(const GdrParams& p, bool bf16, cudaStream_t stream);

struct TreeVerifyParams {
  int R, N, V, greedy;
  float inv_temp;
  const void* logits;         // [R,N,V]
  const float* draft_probs;   // [R,N,V] or nullptr
  const int32_t* token;       // [R,N]
  const int32_t* parent;      // [R,N]
  const int32_t* node_len;    // [R]
  const float* uniform;       // [R,N]
  const float* noise;         // [R,V]
  int32_t* path;              // [R,N]
  int32_t* path_len;          // [R]
  int32_t* next_token;        // [R]
  float* node_logp;           // [R,N]
  int chunk, n_chunks;        // row statistics: tokens per chunk, chunks per row
  // [R,N,n_chunks] {max, sum of 2^(scale (x - max)), first argmax, -} of the logits x,
  // with scale = inv_temp log2 e
  float4* stats;
  int32_t* dev_status;
};
void plan_tree_verify(int R, int N, int V, int num_sms, int* chunk, int* n_chunks);
cudaError_t launch_tree_verify(const TreeVerifyParams& p, bool bf16, cudaStream_t stream);

constexpr int kMaxAppendLayers = 64;
struct TreeAppendParams {
  int R, N, Hkv, D, page_size, num_pages, max_pages, n_layers, elem_bytes;
  const void* k_blk[kMaxAppendLayers];  // each [R,N,Hkv,D]
  const void* v_blk[kMaxAppendLayers];
  void* k_pool[kMaxAppendLayers];       // each [num_pages,Hkv,page_size,D]
  void* v_pool[kMaxAppendLayers];
  const int32_t* page_table;            // [R,max_pages]
  const int32_t* prefix_len;            // [R]
  const int32_t* path;                  // [R,N]
  const int32_t* path_len;              // [R]
  int32_t* dev_status;
};
cudaError_t launch_tree_append(const TreeAppendParams& p, cudaStream_t stream);

constexpr int kMaxTreeNodes = 64;

// Rotation of queries and keys, with or without the append.  Rows r B + t when token_start is
// null, else packed.
struct RotaryParams {
  int R, B, rows, Hq, Hkv, D, rd, interleaved, inverse;
  int page_size, num_pages, max_pages;
  float amplitude;
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;  // elements between rows
  const void* q;               // nullptr: no queries
  const void* k;               // nullptr: no keys
  const void* v;               // append only
  const uint64_t* table;       // [rd / 2] turns a position, 2^64 to a turn
  const int32_t* position;     // [rows] or nullptr
  const int32_t* prefix_len;   // [R] or nullptr
  const int32_t* token_len;    // [R] or nullptr
  const int32_t* parent;       // [R,B] or nullptr
  const int32_t* token_start;  // [R+1] or nullptr
  const int32_t* page_table;   // [R,max_pages], append only
  void* q_out;
  void* k_out;                 // may be nullptr in an append
  void* k_pool;                // nullptr: no append
  void* v_pool;
  int32_t* dev_status;
};
cudaError_t launch_rotary_table(const flare_rotary_freq_desc& d, uint64_t* table,
                                cudaStream_t stream);
cudaError_t launch_rotary(const RotaryParams& p, bool bf16, int num_sms, cudaStream_t stream);

struct TreeLogitsParams {
  int R, N, V, H, max_bias;
  const void* logits;           // [R,N,V]
  const int32_t* history;       // [R,H] or nullptr
  const int32_t* history_len;   // [R]
  const int32_t* output_start;  // [R] or nullptr
  const int32_t* token;         // [R,N] or nullptr
  const int32_t* parent;        // [R,N], with token
  const int32_t* node_len;      // [R] or nullptr
  const float* repetition;      // [R] or nullptr, as the next two
  const float* presence;
  const float* frequency;
  const int32_t* bias_token;    // [R,max_bias] or nullptr
  const float* bias_value;
  const int32_t* bias_len;      // [R]
  const uint32_t* mask;         // [R,N,ceil(V/32)] or nullptr
  void* out;
  int32_t* dev_status;
};
template <typename T>
cudaError_t launch_tree_logits_of(const TreeLogitsParams& p, int num_sms, cudaStream_t stream);
cudaError_t launch_tree_logits(const TreeLogitsParams& p, bool bf16, int num_sms,
                               cudaStream_t stream);

struct BlockNormParams {
  int T, W, G, shared, post, pre, act;  // shared: one weight for all groups, of which there are several
  float eps, alpha;
  int64_t x_stride, gate_stride;
  const void* x;
  const void* gate;      // or nullptr, as the next three
  const void* residual;
  const float* wpost;
  const float* wpre;
  void* y;               // forward: y, h
  void* h;
  const void* dy;        // backward
  const void* dh;
  void* dx;
  void* dgate;
  void* dres;
  float* dwpost;
  float* dwpre;
  float* part;           // [CTAs][2][W] partial weight gradients
};
cudaError_t launch_block_norm(const BlockNormParams& p, bool bf16, int num_sms,
                              cudaStream_t stream);
// The backward pass over rows (T of bf16 or fp32) and how many CTAs it takes at most, on so many
// rows or fewer: each leaves one partial weight gradient.
template <typename T>
cudaError_t launch_block_norm_rows(const BlockNormParams& p, int num_sms, int* ctas, int* cluster,
                                   cudaStream_t stream);
template <typename T>
int block_norm_rows_ctas(int T_rows, int W, bool pre, int num_sms);
int block_norm_bwd_ctas(int T, int W, bool pre, bool bf16, int num_sms);
cudaError_t launch_block_norm_bwd(const BlockNormParams& p, bool bf16, int num_sms,
                                  cudaStream_t stream);

SoftmaxPlan plan_softmax(int R, int B, int Hq, int Hkv, int D, int page_size, int max_pages,
                         bool bf16, int num_sms);
cudaError_t launch_softmax(const SoftmaxParams& p, const SoftmaxPlan& plan, bool bf16,
                           cudaStream_t stream);
cudaError_t launch_softmax_simt(const SoftmaxParams& p, const SoftmaxPlan& plan, bool bf16,
                                cudaStream_t stream);
cudaError_t launch_softmax_tc(const SoftmaxParams& p, const SoftmaxPlan& plan,
                              cudaStream_t stream);
cudaError_t launch_softmax_combine(const SoftmaxParams& p, bool bf16, cudaStream_t stream);
bool softmax_tc_supported(int B, int Hq, int Hkv, int D, int page_size);
cudaError_t launch_append_kv(const SoftmaxParams& p, const int32_t* append_len, void* k_pool,
                             void* v_pool, int elem_bytes, cudaStream_t stream);
cudaError_t launch_debug_wait_timeout(int32_t* status, uint64_t limit_ns, cudaStream_t stream);
cudaError_t launch_gather_prefix(const SoftmaxParams& p, int request, void* k_out, void* v_out,
                                 bool bf16, cudaStream_t stream);

}  // namespace flare
