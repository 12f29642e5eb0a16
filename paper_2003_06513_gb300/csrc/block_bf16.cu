// Block norm's kernels on blocks of __nv_bfloat16 in a stream of the same type.
#include "block.cuh"

template struct patconv::BlockKernels<__nv_bfloat16, __nv_bfloat16>;
