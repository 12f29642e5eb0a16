// Group norm: what the host code (norm.cu) and the kernels' translation units share.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace patconv {

constexpr int kNormThreads = 256;
constexpr unsigned kStatusNormTimeout = 16u;          // pp_device_status: a sample's sums never arrived

struct NormArgs {
    const void *x, *dy;
    int64_t x_pixel, x_sample, dy_pixel, dy_sample;   // strides in elements
    const float *gamma, *beta;
    const float *mean, *rstd;         // [N][G] (backward)
    float *mean_out, *rstd_out;       // (forward)
    void* out;                        // y or dx: dense
    float *dgamma, *dbeta;
    float* parts;                     // pairs: [N][chunks or cluster][sets or channels of a row]
    float* sums;                      // pairs, streamed backward: [N][C], then [N][G]
    uint32_t* counters;               // streamed: tickets, joined samples, [N] parts done, [N] sums ready
    unsigned* status;
    int64_t pixels;
    int N, C, G, cpg, act;
    int cols, rows;                   // vectors of a row a CTA covers, rows it covers at a time
    int chunk;                        // pixels of a CTA at a time
    int spg;                          // sets of channels in a group (forward)
    uint32_t spg_mul, cpg_mul, cols_mul, rows_mul;    // ceil(2^32 / spg) and so on
    float eps;
    int tiles, chunks, ahead, draw, grid;   // streamed: CTAs side by side and stretches down a sample; samples that the
                                      // sums are ahead, items that tickets are; CTAs
    int cluster, slabs, groups;       // resident: CTAs of a unit, slabs of a row, groups of a slab
};

// Streamed kernels: batches of copies under way and one, vectors a thread in a batch (of all inputs).
constexpr int kStreamDepth = 3, kStreamBatch = 8;

inline size_t norm_counters(int N) { return 2 + 2 * (size_t)N; }

// Vectors a thread of a resident kernel holds, of 16 bytes and of 4 or less: the sizes it is compiled for.
constexpr int kHeldWide[] = {2, 4, 8, 16}, kHeldSmall[] = {8, 32};
constexpr int kHeldBackWide[] = {2, 4, 8}, kHeldBackSmall[] = {8, 24};

// Launches of one type's kernels, with V, NS and K of the plan (K 0: streamed).
template <typename T>
struct NormKernels {
    static cudaError_t forward(const NormArgs& a, int V, int NS, int K, cudaStream_t st);
    static cudaError_t backward(const NormArgs& a, int V, int K, cudaStream_t st);
};

// The device's status word (conv.cu), NULL if it cannot be found.
unsigned* device_status_word();

}  // namespace patconv
