// Group norm's kernels on float activations.
#include "norm.cuh"

template struct patconv::NormKernels<float>;
