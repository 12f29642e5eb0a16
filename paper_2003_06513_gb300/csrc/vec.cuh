// Vectors of values in registers, shared by the training side's kernels: loads and stores of 16 bytes and
// narrower, conversion to and from pairs of fp32 values, and the packed arithmetic on such pairs.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>
#include <type_traits>

namespace patconv {
namespace {

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T v[V];
};
template <int V>
constexpr int kPairs = (V + 1) / 2;          // a single value is a pair's first

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load(const T* p) {
    return *reinterpret_cast<const Vec<T, V>*>(p);
}
// a result: not wanted in L2 any longer
template <typename T, int V>
__device__ __forceinline__ void store(T* p, const Vec<T, V>& v) {
    if constexpr (sizeof(T) * V == 16) {
        uint4 w;
        memcpy(&w, &v, 16);
        __stcs(reinterpret_cast<uint4*>(p), w);
    } else {
        *reinterpret_cast<Vec<T, V>*>(p) = v;
    }
}

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__half x) { return __half2float(x); }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }

template <typename T, int V>
__device__ __forceinline__ float2 pair(const Vec<T, V>& v, int i) {
    if constexpr (V == 1) {
        return make_float2(widen(v.v[0]), 0.0f);
    } else if constexpr (sizeof(T) == 4) {
        return make_float2(v.v[2 * i], v.v[2 * i + 1]);
    } else {
        uint32_t w;
        memcpy(&w, &v.v[2 * i], 4);
        if constexpr (std::is_same<T, __half>::value) {
            __half2 h;
            memcpy(&h, &w, 4);
            return __half22float2(h);
        } else {
            return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
        }
    }
}
__device__ __forceinline__ void narrow(float x, float& y) { y = x; }
__device__ __forceinline__ void narrow(float x, __half& y) { y = __float2half_rn(x); }
__device__ __forceinline__ void narrow(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }
template <typename T, int V>
__device__ __forceinline__ void set_pair(Vec<T, V>& v, int i, float2 f) {
    if constexpr (V == 1) {
        narrow(f.x, v.v[0]);
    } else if constexpr (std::is_same<T, __half>::value) {
        const __half2 h = __float22half2_rn(f);
        memcpy(&v.v[2 * i], &h, 4);
    } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        const __nv_bfloat162 h = __float22bfloat162_rn(f);
        memcpy(&v.v[2 * i], &h, 4);
    } else {
        v.v[2 * i] = f.x;
        v.v[2 * i + 1] = f.y;
    }
}

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 neg(float2 a) { return make_float2(-a.x, -a.y); }
__device__ __forceinline__ float2 add(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
// the larger of two, NaN where one of them is (fmaxf takes the other one)
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float approx_rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float approx_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

}  // namespace
}  // namespace patconv
