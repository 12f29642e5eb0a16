// Group norm's kernels on __nv_bfloat16 activations.
#include "norm.cuh"

template struct patconv::NormKernels<__nv_bfloat16>;
