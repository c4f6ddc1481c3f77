// Penalties, biases and masks on logits in fp32.
#include "tree_logits.cuh"

namespace flare {

template cudaError_t launch_tree_logits_of<float>(const TreeLogitsParams&, int, cudaStream_t);

}  // namespace flare
