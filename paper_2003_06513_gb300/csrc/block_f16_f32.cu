// Block norm's kernels on blocks of __half in a stream of fp32.
#include "block.cuh"

template struct patconv::BlockKernels<float, __half>;
