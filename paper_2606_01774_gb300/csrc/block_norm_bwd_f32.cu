// The backward kernels of block norms in fp32.
#include "block_norm_bwd.cuh"

namespace flare {

template cudaError_t launch_block_norm_rows<float>(const BlockNormParams&, int, int*, int*,
                                                cudaStream_t);
template int block_norm_rows_ctas<float>(int, int, bool, int);

}  // namespace flare
