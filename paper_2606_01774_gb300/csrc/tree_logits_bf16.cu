// Penalties, biases and masks on logits in bf16.
#include "tree_logits.cuh"

namespace flare {

template cudaError_t launch_tree_logits_of<__nv_bfloat16>(const TreeLogitsParams&, int, cudaStream_t);

cudaError_t launch_tree_logits(const TreeLogitsParams& p, bool bf16, int num_sms,
                               cudaStream_t stream) {
  if (p.R == 0) return cudaSuccess;
  return bf16 ? launch_tree_logits_of<__nv_bfloat16>(p, num_sms, stream)
              : launch_tree_logits_of<float>(p, num_sms, stream);
}

}  // namespace flare
