// Block norm's kernels on blocks of __half, in a stream of the same type or of fp32.
#include "block.cuh"

template struct patconv::BlockKernels<__half, __half>;
template struct patconv::BlockKernels<float, __half>;
