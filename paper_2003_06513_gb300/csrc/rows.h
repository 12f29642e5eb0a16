// Rows of logits: what the host code and the kernels of a teacher's top logits (top.cu) and of the distillation
// loss (distill.cu, distill_back.cu) share.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "patconv.h"

namespace patconv {

constexpr int kMostKept = 256;                       // classes that are kept of a row at most
constexpr int kMostClasses = 1 << 20;
constexpr int kSMs = 152;

inline int size_of(int dtype) { return dtype == PP_F32 ? 4 : 2; }
inline bool known(int dtype) { return dtype == PP_F32 || dtype == PP_F16 || dtype == PP_BF16; }
inline bool off(const void* p, size_t align) { return reinterpret_cast<uintptr_t>(p) % align != 0; }
// whether two stretches of memory share a byte
inline bool overlap(const void* a, size_t an, const void* b, size_t bn) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return an && bn && x < y + bn && y < x + an;
}
// whether rows may be so far apart
inline bool apart(int64_t rows, int64_t stride, int64_t classes) { return rows <= 1 || (stride >= classes && stride <= (int64_t(1) << 50) / rows); }
// elements from a row's first to the last row's last
inline int64_t row_extent(int64_t rows, int64_t stride, int64_t classes) { return rows ? (rows - 1) * stride + classes : 0; }

struct DistillArgs {
    const void* s;                    // [rows][classes], rows `stride` elements apart
    int64_t stride;
    int rows, classes, kept, value_type;
    const void* values;               // [rows][kept] of value_type
    const int* indices;               // [rows][kept]
    const float* rest;                // [rows] or null
    const int64_t* labels;            // [rows] or null
    float c1, ct, inv_t;              // log2(e), log2(e) / T, 1 / T
    float hard, soft_loss, soft_slope;    // 1 - alpha (0 without labels), alpha T^2, alpha T
    float* loss;                      // [rows]
    float* stats;                     // [rows][5]
    const float* dloss;               // rows `dloss_stride` elements apart
    int64_t dloss_stride;
    void* ds;                         // dense [rows][classes]
    int parts;                        // CTAs of a row
    bool stepwise;                    // whether a row is asked for step by step, not whole
};

cudaError_t distill_forward(const DistillArgs& a, int dtype, cudaStream_t st);
cudaError_t distill_backward(const DistillArgs& a, int dtype, cudaStream_t st);

}  // namespace patconv
