// The backward kernels of block norms in bf16.
#include "block_norm_bwd.cuh"

namespace flare {

template cudaError_t launch_block_norm_rows<__nv_bfloat16>(const BlockNormParams&, int, int*, int*,
                                                        cudaStream_t);
template int block_norm_rows_ctas<__nv_bfloat16>(int, int, bool, int);

}  // namespace flare
