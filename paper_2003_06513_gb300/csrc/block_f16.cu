// Block norm's kernels on blocks of __half in a stream of the same type.
#include "block.cuh"

template struct patconv::BlockKernels<__half, __half>;
