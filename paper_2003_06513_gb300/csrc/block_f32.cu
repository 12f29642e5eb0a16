// Block norm's kernels on blocks of float.
#include "block.cuh"

template struct patconv::BlockKernels<float, float>;
