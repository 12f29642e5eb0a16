// Group norm: what the host code (norm.cu) and the kernels' translation units share.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace patconv {

constexpr int kNormThreads = 256;

struct NormArgs {
    const void *x, *dy;
    int64_t x_pixel, x_sample, dy_pixel, dy_sample;   // strides in elements
    const float *gamma, *beta;
    const float *mean, *rstd;         // [N][G] (backward)
    float *mean_out, *rstd_out;       // (forward)
    void* out;                        // y or dx: dense
    float *dgamma, *dbeta;
    float* parts;                     // pairs: [N][chunks or cluster][sets or channels of a row]
    float* sums;                      // pairs, streamed backward: [N][C] dbeta, dgamma, then [N][G] p, q
    int64_t pixels;
    int N, C, G, cpg, act;
    int cols, rows;                   // vectors of a row a CTA covers, rows it covers at a time
    int chunk, held, quarter;         // pixels of a CTA, vectors of each input that it holds, of a quarter of its rows
    int depth;                        // streamed: vectors of a thread that are asked for at a time
    int spg;                          // sets of channels in a group (forward)
    uint32_t spg_mul, cpg_mul, cols_mul, rows_mul;    // ceil(2^32 / spg) and so on
    float eps;
    int tiles, chunks;                // streamed: CTAs side by side and stretches down a sample
    int cluster, slabs, groups;       // resident: CTAs of a unit (0: streamed), slabs of a row, groups of a slab
};

constexpr int kNormShared = 200 * 1024;               // dynamic shared memory of a CTA at most, beside its static arrays

bool norm_starts_early();             // whether a call's kernels start while the one before ends (norm.cu)

// Launches of one type's kernels, with V and NS of the plan.
template <typename T>
struct NormKernels {
    static cudaError_t forward(const NormArgs& a, int V, int NS, cudaStream_t st);
    static cudaError_t backward(const NormArgs& a, int V, cudaStream_t st);
};

}  // namespace patconv
