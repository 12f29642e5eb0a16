// Kernel parts that top.cu, distill.cu and distill_back.cu share: a row of logits as aligned vectors, groups of
// threads (a warp, or a CTA) that take a row together, and the base-2 exponentials.
#pragma once

#include <climits>
#include <cmath>

#include "rows.h"
#include "vec.cuh"

namespace patconv {
namespace {

constexpr float kNone = -INFINITY;

// A row (or a slice of one) of `count` values from p on, as vectors of W that lie on 16-byte boundaries: places are
// counted from the boundary at or before p, so that value i is at place i + pad and vector v holds places v W to
// v W + W - 1, of which the row has those from pad to end - 1.
template <typename T, int W>
struct Row {
    const T* base;                    // place 0
    int pad, end;
    __device__ __forceinline__ Row(const T* p, int count) {
        pad = W == 1 ? 0 : (int)(reinterpret_cast<uintptr_t>(p) % (W * sizeof(T)) / sizeof(T));
        base = p - pad;
        end = count + pad;
    }
    __device__ __forceinline__ int vectors() const { return (end + W - 1) / W; }
    __device__ __forceinline__ bool whole(int v) const { return v * W >= pad && v * W + W <= end; }
    __device__ __forceinline__ Vec<T, W> at(int v) const { return load<T, W>(base + (int64_t)v * W); }
    // a vector that may lie partly outside the row, where it is -inf: as words, so that the whole ones stay as they are read
    __device__ __forceinline__ Vec<T, W> some(int v) const {
        uint4 w;
        if (whole(v)) {
            w = *reinterpret_cast<const uint4*>(base + (int64_t)v * W);
        } else {
            uint32_t words[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                constexpr int A = W / 4;              // values of a word
                uint32_t bits = 0;
#pragma unroll
                for (int k = 0; k < A; ++k) {
                    const int place = v * W + i * A + k;
                    const T x = place >= pad && place < end ? base[place] : T(kNone);
                    uint32_t b = 0;
                    memcpy(&b, &x, sizeof(T));
                    bits |= b << (16 * k);
                }
                words[i] = bits;
            }
            w = make_uint4(words[0], words[1], words[2], words[3]);
        }
        Vec<T, W> b;
        memcpy(&b, &w, 16);
        return b;
    }
    // the row's vectors from first to last - 1 on their way to L2, all asked for at once
    __device__ __forceinline__ void prefetch(int first, int last) const {
        if (first < last && !whole(first)) ++first;
        if (first < last && !whole(last - 1)) --last;
        if (first < last)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(base + (int64_t)first * W), "r"((last - first) * 16) : "memory");
    }
};

// The threads that take a row together: a warp of several in a CTA (N = 32), or a CTA.
template <int N>
struct Group {
    static constexpr int kWarps = N / 32;
    int lane;                         // of the group
    float* scratch;                   // 2 x kWarps x 8 floats (N > 32)
    int turn = 0;
    __device__ __forceinline__ explicit Group(float* s) : lane(N == 32 ? threadIdx.x % 32 : threadIdx.x), scratch(s) {}
    __device__ __forceinline__ static void sync() {
        if constexpr (N == 32)
            __syncwarp();
        else
            __syncthreads();
    }
    __device__ __forceinline__ static bool any(bool x) {
        if constexpr (N == 32)
            return __any_sync(0xffffffffu, x);
        else
            return __syncthreads_or(x);
    }
    // the group's results of up to 8 values, to every thread, joined in a fixed order; the scratch is used in turns, so
    // that one barrier a call is enough
    template <int K, typename Op>
    __device__ __forceinline__ void join(float (&v)[K], Op op) {
#pragma unroll
        for (int o = 16; o; o >>= 1)
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] = op(v[k], __shfl_xor_sync(0xffffffffu, v[k], o));
        if constexpr (N > 32) {
            float* mine = scratch + turn * kWarps * 8;
            turn ^= 1;
            if (threadIdx.x % 32 == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) mine[threadIdx.x / 32 * 8 + k] = v[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                v[k] = mine[k];
                for (int w = 1; w < kWarps; ++w) v[k] = op(v[k], mine[w * 8 + k]);
            }
        }
    }
    template <int K>
    __device__ __forceinline__ void max(float (&v)[K]) {
        join(v, [](float a, float b) { return fmaxf(a, b); });
    }
    template <int K>
    __device__ __forceinline__ void sum(float (&v)[K]) {
        join(v, [](float a, float b) { return a + b; });
    }
};

// What exponentials are relative to: 2^((x - m) c), c = log2(e) / T, for the largest value m; 0 where there is no value (-inf).
// The difference comes first: x c by itself would leave fp32's range where x is the type's lowest value, as masks have it.
__device__ __forceinline__ float reference(float m) { return m == kNone ? 0.0f : m; }
__device__ __forceinline__ float power(float x, float m, float c) { return approx_exp2((x - m) * c); }
// 2^((a - m) c), 0 where there is no a
__device__ __forceinline__ float factor(float a, float m, float c) { return a == kNone ? 0.0f : approx_exp2((a - m) * c); }

// The largest of values as they come, a NaN above all: packed where two share a register.
template <typename T>
struct Largest;
template <>
struct Largest<float> {
    float m = kNone;
    __device__ __forceinline__ void take(const Vec<float, 4>& v) { m = larger(larger(m, v.v[0]), larger(larger(v.v[1], v.v[2]), v.v[3])); }
    __device__ __forceinline__ float get() const { return m; }
};
template <>
struct Largest<__half> {
    __half2 m = __float2half2_rn(kNone);
    __device__ __forceinline__ void take(const Vec<__half, 8>& v) {
        __half2 h[4];
        memcpy(h, &v, 16);
        m = __hmax2_nan(__hmax2_nan(m, h[0]), __hmax2_nan(__hmax2_nan(h[1], h[2]), h[3]));
    }
    __device__ __forceinline__ float get() const { return larger(__low2float(m), __high2float(m)); }
};
template <>
struct Largest<__nv_bfloat16> {
    __nv_bfloat162 m = __float2bfloat162_rn(kNone);
    __device__ __forceinline__ void take(const Vec<__nv_bfloat16, 8>& v) {
        __nv_bfloat162 h[4];
        memcpy(h, &v, 16);
        m = __hmax2_nan(__hmax2_nan(m, h[0]), __hmax2_nan(__hmax2_nan(h[1], h[2]), h[3]));
    }
    __device__ __forceinline__ float get() const { return larger(__low2float(m), __high2float(m)); }
};
template <typename T, int W>
__device__ __forceinline__ float largest(const Vec<T, W>& v) {
    Largest<T> l;
    l.take(v);
    return l.get();
}

// kept value j of a row, in fp32
__device__ __forceinline__ float value_at(const void* values, int type, int64_t j) {
    if (type == PP_F32) return static_cast<const float*>(values)[j];
    if (type == PP_F16) return __half2float(static_cast<const __half*>(values)[j]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(values)[j]);
}

}  // namespace
}  // namespace patconv
