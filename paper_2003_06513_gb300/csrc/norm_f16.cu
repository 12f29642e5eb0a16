// Group norm's kernels on __half activations.
#include "norm.cuh"

template struct patconv::NormKernels<__half>;
