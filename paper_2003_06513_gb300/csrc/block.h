// Block norm: what the host code (block.cu) and the kernels' translation units share.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace patconv {

constexpr int kBlockEight = 8;                        // channels of a thread
constexpr int kBlockThreads = 256;                    // of a CTA whose rows are of at most a warp
constexpr int kBlockBackThreads = 128;                // in the backward pass: four of them, of 128 registers a thread, on an SM
constexpr int kBlockMost = 4096;                      // channels at most
constexpr int kBlockSums = 5;                         // sums over all rows: weight, bias, post_weight, post_bias, scale

struct BlockArgs {
    const void *x, *b, *dh, *dy;                      // x: the stream before (forward) or after (backward) the block
    int64_t x_pixel, x_sample, b_pixel, b_sample, dh_pixel, dh_sample, dy_pixel, dy_sample;
    const float *post_weight, *post_bias, *scale, *gate, *weight, *bias;
    int post, pre, act;
    float eps, inv_c;
    int rows, C, N;
    int64_t pixels;
    uint32_t pixels_mul;                              // row / pixels = row * pixels_mul >> pixels_shift
    int pixels_shift;
    int threads;                                      // of a row
    int vectors;                                      // of a row
    int ragged;                                       // whether its threads have more channels than it has
    int flat, dense;                                  // whether every tensor's samples follow one another as its pixels do; and those too
    int full;                                         // whether no input is missing
    void *h, *y;                                      // (forward)
    void *dx, *db;                                    // (backward)
    float *dweight, *dbias, *dpost_weight, *dpost_bias, *dscale, *dgate;
    int stretch, ctas;                                // rows of a CTA, and CTAs
    float* sums;                                      // [ctas][kBlockSums][C]
    float* gates;                                     // [ctas][2][C]: of a CTA's first and last sample, where others have rows of it
};

// Launches for a stream of TX and blocks of TB, with V channels to a vector: eight where both are of two bytes, four where one is
// fp32 (vectors of 16 bytes lie side by side), two or one.
template <typename TX, typename TB>
struct BlockKernels {
    static cudaError_t forward(const BlockArgs& a, int V, cudaStream_t st);
    static cudaError_t backward(const BlockArgs& a, int V, cudaStream_t st);
};
// sums of the CTAs' parts (block.cu)
cudaError_t block_join(const BlockArgs& a, cudaStream_t st);
// CTAs of a backward pass, and rows of each
int block_ctas(int64_t rows, int C, int64_t* stretch);

}  // namespace patconv
