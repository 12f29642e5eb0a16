// Block norm's kernels on blocks of __nv_bfloat16 in a stream of fp32.
#include "block.cuh"

template struct patconv::BlockKernels<float, __nv_bfloat16>;
