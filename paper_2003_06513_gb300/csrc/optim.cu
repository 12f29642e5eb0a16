// Operators over many tensors at once, for masked retraining: the gradients' norm and AdamW steps.
//
// The tensors are cut into chunks of kChunk elements; a table in device memory, built once, says where a
// chunk's parameters, states and tap masks are: one reading of 64 bytes, 0.2 % of a step's traffic, before the
// data.  The norm, which needs no more than masks, has a table of its own, of spans of kSpan elements.  The gradients' addresses change from step to step and travel as kernel arguments, so that a step
// is one launch or two however many tensors there are (of up to kMaxGrads, and as many for each kMaxGrads
// beyond).
//
// A tap mask is the packer's own form: nine bits for each 3x3 kernel.  An element that its mask leaves
// out takes no part: its gradient is not used, whatever it is, and its parameter stays.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <cstring>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "patconv.h"

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 256;               // elements that share a scale: a warp's, eight a lane
constexpr int kChunk = kThreads * 8;      // elements of a CTA's chunk: a block a warp, eight a lane
constexpr int kSpan = 8 * kChunk;         // elements that a CTA of the norm's kernel takes at a time
constexpr int kFewGrads = 64, kMaxGrads = 448;   // 448 addresses and the rest are below 4 KB of arguments
constexpr int64_t kMaxNumel = int64_t(1) << 40;

struct Tensor {                           // what the handle keeps of one on the host
    int64_t numel, state;                 // state: its first element in the states
    int grad_dtype;
    bool masked;
};

struct alignas(64) Chunk {                // of the device table: consecutive elements of one tensor
    float* param;                         // of the first one, here and below
    uint16_t* copy;
    const uint16_t* taps;                 // of its 3x3 kernel; NULL: no mask
    int64_t state, first;                 // its place in the states and in the tensor
    uint32_t tensor;
    uint16_t count;                       // elements, 1 to kChunk
    uint8_t tap, grad_dtype;              // tap: its place in its 3x3 kernel
    float decay;
};
static_assert(sizeof(Chunk) == 64, "a line's half");

struct Span {                             // the norm's table: up to kSpan consecutive elements of one tensor
    const uint16_t* taps;                 // as a chunk's
    int64_t first;
    uint32_t tensor, count;
    uint32_t tap, grad_dtype;
};

template <int N>
struct Grads {
    const void* at[N];
};

}  // namespace

struct pp_tensors {
    std::vector<Tensor> tensors;
    std::vector<uint32_t> first_chunk;    // chunks of the tensors before each (whole launches matter), and of all; none without params
    std::vector<uint32_t> first_span;     // the same of spans
    std::vector<uint32_t> masked_end;     // per launch: the end of its chunks of tensors with masks, which come first
    std::vector<uint8_t> image;           // chunks | spans | counters and partial sums (zero)
    size_t off_spans = 0, off_sums = 0;
    int64_t state_elements = 0;
    int copy_dtype = PP_F16;
    bool has_params = false;
    unsigned char* dev = nullptr;
};

namespace {

constexpr int kSMs = 152;
constexpr int kSumCtas = kSMs * 5;        // most CTAs of the norm's kernel
constexpr unsigned kCounters = 64;        // its CTAs report to one each of these, and the last of each to one more
constexpr size_t kCounterBytes = 512;

struct Vec8 {
    float v[8];
};

__device__ __forceinline__ Vec8 load8(const float* p) {
    Vec8 r;
    asm volatile("ld.global.L1::no_allocate.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(r.v[0]), "=f"(r.v[1]), "=f"(r.v[2]), "=f"(r.v[3]), "=f"(r.v[4]), "=f"(r.v[5]), "=f"(r.v[6]),
                   "=f"(r.v[7])
                 : "l"(p)
                 : "memory");
    return r;
}
__device__ __forceinline__ void store8(float* p, const Vec8& r) {
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(r.v[0]), "f"(r.v[1]), "f"(r.v[2]),
                 "f"(r.v[3]), "f"(r.v[4]), "f"(r.v[5]), "f"(r.v[6]), "f"(r.v[7])
                 : "memory");
}
// Pairs of values, two to an instruction.  A product of mul2 and a sum of add2 that follows it may become one fused
// operation, whatever rounding is written there: where both have to round, the sum is an fma2 (moments2).
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{.reg .b64 x, y, z; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mul.rn.f32x2 z, x, y; mov.b64 {%0, %1}, z;}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{.reg .b64 x, y, z; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; add.rn.f32x2 z, x, y; mov.b64 {%0, %1}, z;}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 widen(uint32_t w, int dtype) {
    if (dtype == PP_F16) {
        __half2 h;
        memcpy(&h, &w, 4);
        return __half22float2(h);
    }
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ float widen1(const void* p, int64_t i, int dtype) {
    if (dtype == PP_F32) return static_cast<const float*>(p)[i];
    const uint16_t w = static_cast<const uint16_t*>(p)[i];
    return widen(w, dtype).x;
}
__device__ __forceinline__ uint16_t narrow1(float f, int dtype) {
    if (dtype == PP_F16) return __half_as_ushort(__float2half_rn(f));
    return __bfloat16_as_ushort(__float2bfloat16_rn(f));
}

// whether eight-element accesses from a tensor's start are aligned
__device__ __forceinline__ bool wide_grad(const void* g, int dtype) {
    return (reinterpret_cast<uintptr_t>(g) & (dtype == PP_F32 ? 31 : 15)) == 0;
}

// Which of the eight elements from element `le` of a chunk on take part: in the tensor (n of them) and kept
// by its mask.  Eight elements touch two 3x3 kernels at most.
__device__ __forceinline__ uint32_t kept8(const uint16_t* taps, uint32_t tap, uint32_t count, uint32_t le, int n) {
    if (n <= 0) return 0;
    const uint32_t in = n >= 8 ? 0xFFu : (1u << n) - 1;
    if (!taps) return in;
    const uint32_t local = tap + le, k = local / 9, r = local - 9 * k;
    const uint32_t a = taps[k] & 0x1FFu;
    const uint32_t b = 9 * (k + 1) < tap + count ? taps[k + 1] & 0x1FFu : 0;
    return ((a | b << 9) >> r) & in;
}
// elements of the tensor among the eight from element `le` of a chunk on
__device__ __forceinline__ int in_chunk(uint32_t count, uint32_t le) { return max(0, min(8, (int)count - (int)le)); }

// ------------------------------------------------------------------------------------- the norm

// Eight gradients as they lie in memory.
template <int GRAD>
struct RawGrad {
    uint4 w[GRAD == PP_F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void* g, int64_t e) {
        if constexpr (GRAD == PP_F32) {
            const Vec8 x = load8(static_cast<const float*>(g) + e);
            memcpy(w, &x, 32);
        } else {
            w[0] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(g) + e));
        }
    }
    __device__ __forceinline__ uint32_t word(int i) const {
        const uint4 q = w[0];
        return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w;
    }
    __device__ __forceinline__ float2 pair(int i) const {
        const uint4 q = w[GRAD == PP_F32 ? i / 2 : 0];
        if constexpr (GRAD == PP_F32)
            return i % 2 ? make_float2(__uint_as_float(q.z), __uint_as_float(q.w)) : make_float2(__uint_as_float(q.x), __uint_as_float(q.y));
        return widen(word(i), GRAD);
    }
};
// A sum of positive terms and what its roundings have lost.
struct LongSum {
    float sum = 0.0f, lost = 0.0f;
    __device__ __forceinline__ void add(float x) {
        const float t = sum + x;
        lost += x - (t - sum);
        sum = t;
    }
};

// Sum of (g f)^2 for a factor f over the spans that a CTA takes, U eights a thread at a time: their gradients
// are asked for before the first is used, and with them the next ones' masks and the next span's entry.
// WIDE: fp32 gradients among them; SCALED: f is not 1.
template <int N, bool WIDE, bool SCALED>
__device__ __forceinline__ float span_squares(const Span* spans, uint32_t begin, uint32_t end, uint32_t t0,
                                              const Grads<N>& grads, float factor, float* smem) {
    constexpr int U = WIDE ? 2 : 4;
    LongSum sum;
    const uint32_t le = threadIdx.x * 8;
    uint32_t c = begin + blockIdx.x;
    Span next{};
    if (c < end) next = spans[c];
#pragma unroll 1
    for (; c < end; c += gridDim.x) {
        const Span sp = next;
        if (c + gridDim.x < end) next = spans[c + gridDim.x];
        const char* base = static_cast<const char*>(grads.at[sp.tensor - t0]);
        if (!base) continue;
        const uint32_t dtype = sp.grad_dtype, count = sp.count, size = WIDE && dtype == PP_F32 ? 4 : 2;
        const bool wide = wide_grad(base, dtype);
        const char* g = base + (sp.first + le) * size;
        uint32_t from = 0;
        if (wide && !sp.taps && !SCALED) {        // whole eights, all of them kept
#pragma unroll 1
            for (; from + U * kChunk <= count; from += U * kChunk, g += U * kChunk * size) {
                uint4 raw[U][WIDE ? 2 : 1];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (WIDE && dtype == PP_F32) {
                        const Vec8 v = load8(reinterpret_cast<const float*>(g) + u * kChunk);
                        memcpy(raw[u], &v, WIDE ? 32 : 16);
                    } else {
                        raw[u][0] = __ldcs(reinterpret_cast<const uint4*>(g + u * kChunk * 2));
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float2 s = make_float2(0.0f, 0.0f);
                    const auto take = [&](const uint4& w, bool f32) {
                        const uint32_t k[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int i = 0; i < 4; i += f32 ? 2 : 1) {
                            const float2 x = f32 ? make_float2(__uint_as_float(k[i]), __uint_as_float(k[i + 1 < 4 ? i + 1 : i])) : widen(k[i], dtype);
                            s = fma2(x, x, s);
                        }
                    };
                    if (WIDE && dtype == PP_F32) {
                        take(raw[u][0], true);
                        take(raw[u][WIDE ? 1 : 0], true);
                    } else {
                        take(raw[u][0], false);
                    }
                    sum.add(s.x + s.y);
                }
            }
        }
        if (from >= count) continue;
        uint32_t keep[U];
        const auto masks = [&](uint32_t from) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t e = from + u * kChunk + le;
                keep[u] = kept8(sp.taps, sp.tap, count, e, in_chunk(count, e));
            }
        };
        masks(from);
#pragma unroll 1
        for (; from < count; from += U * kChunk, g += U * kChunk * size) {
            uint4 raw[U][WIDE ? 2 : 1];
            uint32_t now[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                now[u] = keep[u];
                if (!now[u] || !wide || from + u * kChunk + le + 8 > count) continue;
                if (WIDE && dtype == PP_F32) {
                    const Vec8 v = load8(reinterpret_cast<const float*>(g) + u * kChunk);
                    memcpy(raw[u], &v, WIDE ? 32 : 16);
                } else {
                    raw[u][0] = __ldcs(reinterpret_cast<const uint4*>(g + u * kChunk * 2));
                }
            }
            if (from + U * kChunk < count) masks(from + U * kChunk);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!now[u]) continue;
                float x[8];
                if (!wide || from + u * kChunk + le + 8 > count) {       // a tensor's end, or one that is not aligned
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = now[u] >> i & 1 ? widen1(g + u * kChunk * size, i, dtype) : 0.0f;
                } else if (WIDE && dtype == PP_F32) {
                    memcpy(x, raw[u], WIDE ? 32 : 16);
                } else {
                    const uint32_t w[4] = {raw[u][0].x, raw[u][0].y, raw[u][0].z, raw[u][0].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 f = widen(w[i], dtype);
                        x[2 * i] = f.x;
                        x[2 * i + 1] = f.y;
                    }
                }
                float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float2 y = make_float2(x[2 * i], x[2 * i + 1]);
                    if (SCALED) y = mul2(y, both(factor));
                    y = make_float2(now[u] >> (2 * i) & 1 ? y.x : 0.0f, now[u] >> (2 * i + 1) & 1 ? y.y : 0.0f);
                    s = fma2(y, y, s);
                }
                sum.add(s.x + s.y);
            }
        }
    }
    float s = sum.lost == sum.lost ? sum.sum + sum.lost : sum.sum;        // infinity has no rounding
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    __syncthreads();
    if (threadIdx.x % 32 == 0) smem[threadIdx.x / 32] = s;
    __syncthreads();
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) s += smem[i];
    return s;
}

// Measured on a GB300 (a copy moves 6.67 TB/s), gradients in memory: 56.6 M bf16 gradients without masks 24 us
// (4.6 TB/s, 17 us of it the reading; the rest is the launch and the last CTA's sum); ResNet-50's 3x3 layers, a
// kernel in 0.4 kept, fp32, 16 us: 42 MB of traffic in whole 64-byte pieces, 6 us of it the reading, the rest the
// chain of a span's entry, masks and four readings and that sum.  With spans of 2048 elements the first took 36 us.
//
// Partial sums of squares, one a CTA, and in the last CTA to finish of the call's last launch their sum
// in 64 bits, the norm and the clip factor.  Squares that leave fp32's range (a sum below 2^-80, where
// they may have been rounded away, or above 2^120) are summed again with the gradients times 2^64 or
// 2^-64, so that the norm holds over fp32's whole range of gradients.
template <int N, bool WIDE>
__global__ void __launch_bounds__(kThreads, WIDE ? 5 : 4) grad_norm_kernel(const Span* spans, uint32_t begin, uint32_t end, uint32_t t0,
                                                                Grads<N> grads, double* sums, unsigned* counter,
                                                                unsigned first_sum, unsigned all_sums, float max_norm,
                                                                float* out) {
    __shared__ float smem[kThreads / 32];
    __shared__ double dsum[kThreads / 32];
    __shared__ bool last;
    float s = span_squares<N, WIDE, false>(spans, begin, end, t0, grads, 1.0f, smem);
    double total = s;
    if (!(s >= 0x1p-80f && s <= 0x1p120f)) {      // uniform over the CTA
        const bool small = s < 0x1p-80f;
        s = span_squares<N, WIDE, true>(spans, begin, end, t0, grads, small ? 0x1p64f : 0x1p-64f, smem);
        total = (double)s * (small ? 0x1p-128 : 0x1p128);
    }
    if (threadIdx.x == 0) {
        // thousands of CTAs at one counter would take 10 ns each; the last of all is the last of its counter's
        const unsigned me = first_sum + blockIdx.x, own = me % kCounters;
        sums[me] = total;
        __threadfence();
        last = atomicAdd(counter + 1 + own, 1) == (all_sums - own + kCounters - 1) / kCounters - 1;
        if (last) {
            counter[1 + own] = 0;                 // for the next call
            __threadfence();
            last = atomicAdd(counter, 1) == min(all_sums, kCounters) - 1;
        }
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double d = 0.0;
#pragma unroll 8
    for (unsigned i = threadIdx.x; i < all_sums; i += kThreads) d += __ldcg(sums + i);
#pragma unroll
    for (int o = 16; o; o >>= 1) d += __shfl_down_sync(0xffffffffu, d, o);
    if (threadIdx.x % 32 == 0) dsum[threadIdx.x / 32] = d;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kThreads / 32; ++i) d += dsum[i];
        const float norm = (float)sqrt(d);
        // no clipping where max_norm is infinite, of an infinite norm either; NaN stays NaN
        const float f = max_norm == INFINITY && norm == INFINITY ? 1.0f : max_norm / (norm + 1e-6f);
        out[0] = norm;
        out[1] = f > 1.0f ? 1.0f : f;
        *counter = 0;                             // for the next call
    }
}

// ------------------------------------------------------------------------------------- AdamW

struct AdamArgs {
    float lr, step_size, b1, b2, c1, c2, inv_bc2, eps;   // step_size = lr / (1 - b1^t), c = 1 - b
    float one;                                           // 1, which the compiler is not told
    uint32_t key;
    int copy_dtype;
    const float* grad_scale;
    void *m, *v;
    float *m_scale, *v_scale;
};

__device__ __forceinline__ float approx_sqrt(float x) {
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float approx_rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The states' arithmetic rounds every product and sum by itself: an 8-bit state then depends on the
// formula alone, and not on which of the kernels' paths an element takes or on how a compiler contracts it.
// The packed form has no instructions that are kept apart: there a sum x + y is x * one + y, one rounding of
// the sum of two rounded products, since `one` is 1 and x's own product cannot become a part of it.  It costs what
// the packed sum does.  m and v come as values times mb and vb: an 8-bit state's code and its scale times b, a
// product by a power of two being exact.
__device__ __forceinline__ void moments(float g, float& m, float& v, float mb, float vb, const AdamArgs& a) {
    m = __fadd_rn(__fmul_rn(m, mb), __fmul_rn(g, a.c1));
    v = __fadd_rn(__fmul_rn(v, vb), __fmul_rn(__fmul_rn(g, g), a.c2));
}
__device__ __forceinline__ void moments2(float2 g, float2& m, float2& v, float mb, float vb, const AdamArgs& a) {
    m = fma2(mul2(m, both(mb)), both(a.one), mul2(g, both(a.c1)));
    v = fma2(mul2(v, both(vb)), both(a.one), mul2(mul2(g, g), both(a.c2)));
}
// 2^-126 keeps the root in fp32's normal range, where the approximations flush nothing: a root below
// 2^-63 is far below any eps in use, and with eps = 0 it makes 0 / 0 zero.
__device__ __forceinline__ float stepped(float p, float m, float v, float shrink, const AdamArgs& a) {
    const float den = approx_sqrt(fmaf(v, a.inv_bc2, 0x1p-126f)) + a.eps;
    return fmaf(-a.step_size, m * approx_rcp(den), p * shrink);
}

__device__ __forceinline__ float2 stepped2(float2 p, float2 m, float2 v, float shrink, const AdamArgs& a) {
    const float2 w = fma2(v, both(a.inv_bc2), both(0x1p-126f));
    const float2 den = add2(make_float2(approx_sqrt(w.x), approx_sqrt(w.y)), both(a.eps));
    const float2 u = mul2(m, make_float2(approx_rcp(den.x), approx_rcp(den.y)));
    return fma2(both(-a.step_size), u, mul2(p, both(shrink)));
}

__host__ __device__ inline uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0xCBBB9D5Du;
    x ^= x >> 15;
    x *= 0x629A292Bu;
    return x ^ x >> 16;
}

// A block's scale: the power of two that brings its largest magnitude into (224, 448], e4m3's top.
__device__ __forceinline__ float block_scale(uint32_t largest) {
    if (!largest) return 1.0f;
    const int field = (int)((largest + 0x1FFFFFu) >> 23) - 8;    // 1.75 2^k and below have exponent k
    return __uint_as_float((uint32_t)(field < 1 ? 1 : field) << 23);
}

// the reciprocal of a power of two between 2^-126 and 2^126
__device__ __forceinline__ float inverse_scale(float scale) { return __uint_as_float((254u << 23) - __float_as_uint(scale)); }

// A finite value over its block's scale, rounded to one of its two neighbours in e4m3 by the dither: 16
// random bits, then a half, in the place of the bits below the format's three, which are filled up by it
// and cut off.  Below 2^-6 the format's grid is that of [2^-6, 2^-5), so 2^-6 is added for the cut.
__device__ __forceinline__ float rounded(float t, uint32_t dither) {      // either sign
    const float small = fabsf(t) < 0x1p-6f ? copysignf(0x1p-6f, t) : 0.0f;
    return __uint_as_float((__float_as_uint(__fadd_rn(t, small)) + dither) & 0xFFF00000u) - small;
}
__device__ __forceinline__ float rounded_up(float t, uint32_t dither) {   // not negative; above zero stays so
    const float small = t < 0x1p-6f ? 0x1p-6f : 0.0f;
    const float w = __uint_as_float((__float_as_uint(__fadd_rn(t, small)) + dither) & 0xFFF00000u) - small;
    return t > 0.0f ? fmaxf(w, 0x1p-9f) : w;
}
__device__ __forceinline__ float cut(float t, uint32_t dither) { return __uint_as_float((__float_as_uint(t) + dither) & 0xFFF00000u); }
__device__ __forceinline__ float2 rounded2(float2 t, uint32_t dx, uint32_t dy) {
    const float2 small = make_float2(fabsf(t.x) < 0x1p-6f ? copysignf(0x1p-6f, t.x) : 0.0f,
                                     fabsf(t.y) < 0x1p-6f ? copysignf(0x1p-6f, t.y) : 0.0f);
    t = add2(t, small);
    return add2(make_float2(cut(t.x, dx), cut(t.y, dy)), make_float2(-small.x, -small.y));
}
__device__ __forceinline__ float2 rounded_up2(float2 t, uint32_t dx, uint32_t dy) {
    const float2 small = make_float2(t.x < 0x1p-6f ? 0x1p-6f : 0.0f, t.y < 0x1p-6f ? 0x1p-6f : 0.0f);
    const float2 u = add2(t, small), w = add2(make_float2(cut(u.x, dx), cut(u.y, dy)), make_float2(-small.x, -small.y));
    return make_float2(t.x > 0.0f ? fmaxf(w.x, 0x1p-9f) : w.x, t.y > 0.0f ? fmaxf(w.y, 0x1p-9f) : w.y);
}
__device__ __forceinline__ uint32_t dither_m(uint32_t y) { return (y << 4 & 0xFFFF0u) | 8; }
__device__ __forceinline__ uint32_t dither_v(uint32_t y) { return (y >> 12 & 0xFFFF0u) | 8; }

// One hash for eight consecutive elements, times an odd constant for each: the first 32 bits of the
// fractions of the square roots of 2 to 19, made odd (mix has those of 23 and 29).
__device__ __forceinline__ uint32_t hash8(int64_t state, uint32_t key) {
    return mix((uint32_t)(state >> 3) * 0x9E3779B1u ^ key);
}
__device__ __forceinline__ uint32_t odd(int i) {
    constexpr uint32_t c[8] = {0x6A09E667u, 0xBB67AE85u, 0x3C6EF373u, 0xA54FF53Bu,
                               0x510E527Fu, 0x9B05688Du, 0x1F83D9ABu, 0x5BE0CD19u};
    return c[i];
}
__device__ __forceinline__ uint32_t own_bits(uint32_t h, uint32_t factor) {
    const uint32_t y = h * factor;
    return y ^ y >> 15;
}

// larger magnitude; NaN if either is NaN
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}

__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
}
__device__ __forceinline__ void unpack4(uint32_t w, float* out) {
    const __half2 a = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xFFFFu), __NV_E4M3));
    const __half2 b = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3));
    const float2 x = __half22float2(a), y = __half22float2(b);
    out[0] = x.x;
    out[1] = x.y;
    out[2] = y.x;
    out[3] = y.y;
}
__device__ __forceinline__ float unpack1(uint8_t w) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(w, __NV_E4M3)));
}
__device__ __forceinline__ uint8_t pack1(float x) { return __nv_cvt_float_to_fp8(x, __NV_SATFINITE, __NV_E4M3); }

// The block's scale from each lane's values.  Where one of them is not finite (a warp's rare case) the
// scale is the others', and `spoilt` says which of the lane's those are: they are stored as NaN.
template <int K>
__device__ __forceinline__ float warp_scale(const float (&x)[K], uint32_t& spoilt) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < K; ++i) top = larger(top, x[i]);
    uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
    spoilt = 0;
    if (bits >= 0x7F800000u) {
        uint32_t fine = 0;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
            if (b < 0x7F800000u)
                fine = max(fine, b);
            else
                spoilt |= 1u << i;
        }
        bits = __reduce_max_sync(0xffffffffu, fine);
    }
    return block_scale(bits);
}
template <int K>
__device__ __forceinline__ void spoil(float (&x)[K], uint32_t spoilt) {
    if (!spoilt) return;
#pragma unroll
    for (int i = 0; i < K; ++i)
        if (spoilt >> i & 1) x[i] = NAN;
}

// e: of the chunk, here and below
__device__ __forceinline__ void store_copy(const Chunk& t, uint32_t e, float p, int dtype) {
    t.copy[e] = narrow1(p, dtype);
}

// A block of any tensor, eight consecutive elements a lane, of which those in `keep` take part: the ends of
// tensors, tensors that are not aligned, masks that keep most of a block.
template <int BITS>
__device__ __noinline__ void any_block(const Chunk t, const void* gp, uint32_t e, uint32_t keep, float gs, float shrink,
                                       const AdamArgs a) {
    const int64_t s = t.state + e;
    float m[8] = {}, v[8] = {}, mb = a.b1, vb = a.b2;
    if (BITS == 8) {
        mb *= a.m_scale[s / kBlock];
        vb *= a.v_scale[s / kBlock];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (!(keep >> i & 1)) continue;
        if constexpr (BITS == 8) {
            m[i] = unpack1(static_cast<const uint8_t*>(a.m)[s + i]);
            v[i] = unpack1(static_cast<const uint8_t*>(a.v)[s + i]);
        } else {
            m[i] = static_cast<const float*>(a.m)[s + i];
            v[i] = static_cast<const float*>(a.v)[s + i];
        }
        moments(__fmul_rn(widen1(gp, e + i, t.grad_dtype), gs), m[i], v[i], mb, vb, a);
        const float p = stepped(t.param[e + i], m[i], v[i], shrink, a);
        t.param[e + i] = p;
        if (t.copy) store_copy(t, e + i, p, a.copy_dtype);
        if constexpr (BITS == 32) {
            static_cast<float*>(a.m)[s + i] = m[i];
            static_cast<float*>(a.v)[s + i] = v[i];
        }
    }
    if (BITS == 32) return;
    uint32_t spoilt_m, spoilt_v;
    const float ms = warp_scale(m, spoilt_m), vs = warp_scale(v, spoilt_v), im = inverse_scale(ms), iv = inverse_scale(vs);
    const uint32_t h = hash8(s, a.key);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (!(keep >> i & 1)) continue;
        const uint32_t y = own_bits(h, odd(i));
        static_cast<uint8_t*>(a.m)[s + i] = pack1(spoilt_m >> i & 1 ? NAN : rounded(m[i] * im, dither_m(y)));
        static_cast<uint8_t*>(a.v)[s + i] = pack1(spoilt_v >> i & 1 ? NAN : rounded_up(v[i] * iv, dither_v(y)));
    }
    if (threadIdx.x % 32 == 0) {
        a.m_scale[s / kBlock] = ms;
        a.v_scale[s / kBlock] = vs;
    }
}

// A whole block of an aligned tensor without a mask, eight consecutive elements a lane.
template <int BITS, int GRAD>
__device__ __forceinline__ void dense_block(const Chunk& t, const void* gp, uint32_t e, float gs, float shrink, const AdamArgs& a) {
    const int64_t s = t.state + e;
    float m[8], v[8], mb = a.b1, vb = a.b2;
    uint2 m8, v8;
    RawGrad<GRAD> g;
    if constexpr (BITS == 8) {
        m8 = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.m) + s));
        v8 = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.v) + s));
        mb *= a.m_scale[s / kBlock];
        vb *= a.v_scale[s / kBlock];
    } else {
        const Vec8 x = load8(static_cast<const float*>(a.m) + s), y = load8(static_cast<const float*>(a.v) + s);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = x.v[i];
            v[i] = y.v[i];
        }
    }
    g.load(gp, e);
    Vec8 p = load8(t.param + e);
    if constexpr (BITS == 8) {
        unpack4(m8.x, m);
        unpack4(m8.y, m + 4);
        unpack4(v8.x, v);
        unpack4(v8.y, v + 4);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 mi = make_float2(m[2 * i], m[2 * i + 1]), vi = make_float2(v[2 * i], v[2 * i + 1]);
        moments2(mul2(g.pair(i), both(gs)), mi, vi, mb, vb, a);
        const float2 pi = stepped2(make_float2(p.v[2 * i], p.v[2 * i + 1]), mi, vi, shrink, a);
        m[2 * i] = mi.x, m[2 * i + 1] = mi.y, v[2 * i] = vi.x, v[2 * i + 1] = vi.y, p.v[2 * i] = pi.x, p.v[2 * i + 1] = pi.y;
    }
    store8(t.param + e, p);
    if (t.copy) {
#pragma unroll
        for (int i = 0; i < 8; ++i) store_copy(t, e + i, p.v[i], a.copy_dtype);
    }
    if constexpr (BITS == 32) {
        Vec8 x, y;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x.v[i] = m[i];
            y.v[i] = v[i];
        }
        store8(static_cast<float*>(a.m) + s, x);
        store8(static_cast<float*>(a.v) + s, y);
    } else {
        uint32_t spoilt_m, spoilt_v;
        const float ms = warp_scale(m, spoilt_m), vs = warp_scale(v, spoilt_v);
        const float2 im = both(inverse_scale(ms)), iv = both(inverse_scale(vs));
        const uint32_t h = hash8(s, a.key);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = own_bits(h, odd(2 * i)), y = own_bits(h, odd(2 * i + 1));
            const float2 mi = rounded2(mul2(make_float2(m[2 * i], m[2 * i + 1]), im), dither_m(x), dither_m(y));
            const float2 vi = rounded_up2(mul2(make_float2(v[2 * i], v[2 * i + 1]), iv), dither_v(x), dither_v(y));
            m[2 * i] = mi.x, m[2 * i + 1] = mi.y, v[2 * i] = vi.x, v[2 * i + 1] = vi.y;
        }
        spoil(m, spoilt_m);
        spoil(v, spoilt_v);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.m) + s) = make_uint2(pack4(m[0], m[1], m[2], m[3]), pack4(m[4], m[5], m[6], m[7]));
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.v) + s) = make_uint2(pack4(v[0], v[1], v[2], v[3]), pack4(v[4], v[5], v[6], v[7]));
        if (threadIdx.x % 32 == 0) {
            a.m_scale[s / kBlock] = ms;
            a.v_scale[s / kBlock] = vs;
        }
    }
}

// A tensor with a mask.  A pruned layer keeps a tenth to a half of its elements, all over a block: the warp
// lists them, and its lanes take the listed ones in turn, so that the arithmetic is done for kept elements
// only.  The others' states are zero and stay so.  Whole vectors with selects in their place took 43 us a step over
// VGG-16's layers with 8-bit states at a kernel in 0.3 kept, lists 35; with all kernels kept 45 and 48.

// Lists a block's kept elements (eight a lane, their bits in `keep`); returns how many there are.
__device__ __forceinline__ int list_kept(uint32_t keep, uint8_t* list) {
    const int lane = threadIdx.x % 32;
    uint32_t upto = __popc(keep);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t below = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += below;
    }
    uint8_t* to = list + (upto - __popc(keep));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (keep >> i & 1) *to++ = (uint8_t)(lane * 8 + i);
    return __shfl_sync(0xffffffffu, upto, 31);
}

// What the lanes read of a block's `count` listed elements, R rounds of 32 at most; lanes past the last read
// it again.
template <int BITS, int R>
struct Listed {
    float p[R], m[R], v[R], ms, vs;
    uint32_t g[R];                                // as they lie in memory, and m and v of 8 bits too: a conversion would
                                                  // wait for a round's values before the next round is asked for
    static_assert(R <= 4, "a byte of `elements` a round");
    uint32_t elements;                            // of the block, the lane's of every round
    __device__ __forceinline__ uint32_t element(int r) const { return __byte_perm(elements, 0, 0x4440 | r); }
    // e0: the block's first element
    __device__ __forceinline__ void load(const Chunk& t, const void* gp, uint32_t e0, const uint8_t* list, int count,
                                         const AdamArgs& a) {
        const int64_t s0 = t.state + e0;
        const float* params = t.param + e0;
        const bool g32 = t.grad_dtype == PP_F32;
        ms = vs = 1.0f;
        elements = 0;
        if constexpr (BITS == 8) {
            ms = a.m_scale[s0 / kBlock];
            vs = a.v_scale[s0 / kBlock];
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = v[r] = 0.0f;
            if (r * 32 >= count) continue;        // the whole warp
            const uint32_t el = list[min(r * 32 + (int)(threadIdx.x % 32), count - 1)];
            elements |= el << (8 * r);
            if (g32)
                g[r] = (static_cast<const uint32_t*>(gp) + e0)[el];
            else
                g[r] = (static_cast<const uint16_t*>(gp) + e0)[el];
            p[r] = params[el];
            if constexpr (BITS == 8) {
                m[r] = __uint_as_float((static_cast<const uint8_t*>(a.m) + s0)[el]);
                v[r] = __uint_as_float((static_cast<const uint8_t*>(a.v) + s0)[el]);
            } else {
                m[r] = (static_cast<const float*>(a.m) + s0)[el];
                v[r] = (static_cast<const float*>(a.v) + s0)[el];
            }
        }
    }
    __device__ __forceinline__ void step(const Chunk& t, uint32_t e0, int count, float gs, float shrink,
                                         const AdamArgs& a) {
        const int64_t s0 = t.state + e0;
        const int lane = threadIdx.x % 32;
        float* params = t.param + e0;
        __syncwarp();                             // all lanes have read what the last one writes
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r * 32 >= count) continue;
            if constexpr (BITS == 8) {
                m[r] = unpack1((uint8_t)__float_as_uint(m[r]));
                v[r] = unpack1((uint8_t)__float_as_uint(v[r]));
            }
            const float gr = t.grad_dtype == PP_F32 ? __uint_as_float(g[r]) : widen(g[r], t.grad_dtype).x;
            moments(__fmul_rn(gr, gs), m[r], v[r], a.b1 * ms, a.b2 * vs, a);
            const float to = stepped(p[r], m[r], v[r], shrink, a);
            if (r * 32 + lane < count) {
                const uint32_t el = element(r);
                params[el] = to;
                if (t.copy) store_copy(t, e0 + el, to, a.copy_dtype);
                if constexpr (BITS == 32) {
                    (static_cast<float*>(a.m) + s0)[el] = m[r];
                    (static_cast<float*>(a.v) + s0)[el] = v[r];
                }
            }
        }
        if constexpr (BITS == 32) return;
        uint32_t spoilt_m, spoilt_v;
        ms = warp_scale(m, spoilt_m);
        vs = warp_scale(v, spoilt_v);
        const float im = inverse_scale(ms), iv = inverse_scale(vs);
        uint32_t factor = 0;                      // lane i < 8 has odd(i)
#pragma unroll
        for (int i = 0; i < 8; ++i) factor = lane == i ? odd(i) : factor;
        const uint32_t hash = hash8(s0 + 8 * lane, a.key);            // of the lane's eight elements of the block
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r * 32 >= count) continue;
            const uint32_t el = element(r);
            const uint32_t y = own_bits(__shfl_sync(0xffffffffu, hash, el >> 3), __shfl_sync(0xffffffffu, factor, el & 7));
            m[r] = rounded(m[r] * im, dither_m(y));
            v[r] = rounded_up(v[r] * iv, dither_v(y));
        }
        spoil(m, spoilt_m);
        spoil(v, spoilt_v);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r * 32 + lane >= count) continue;
            const uint32_t el = element(r);
            (static_cast<uint8_t*>(a.m) + s0)[el] = pack1(m[r]);
            (static_cast<uint8_t*>(a.v) + s0)[el] = pack1(v[r]);
        }
        if (lane == 0) {
            a.m_scale[s0 / kBlock] = ms;
            a.v_scale[s0 / kBlock] = vs;
        }
    }
};

// A chunk a CTA, a block of 256 elements a warp: many light CTAs hide the tables' latency better than few
// that look ahead.  MASKED: for chunks of tensors with masks, whose chain of readings (chunk, masks, data) wants more of them on an SM: with six CTAs
// the pruned layers below take 5 % less time than with five; eight leave too few registers.
//
// Measured on a GB300 (a copy moves 6.67 TB/s), states and parameters in memory:
//     24 dense layers, 56.6 M elements, fp32 gradients, 8-bit states   145 us, 6.3 TB/s: memory
//     ResNet-50's 3x3 layers, dense, fp32 gradients and states          50 us, 6.3 TB/s: memory
//     VGG-16's, a kernel in 0.3 kept, fp32 gradients and states         49 us: the kept elements' 1.2 TB/s are
//         4.9 TB/s of memory traffic, since what is read is whole 64-byte pieces with any kept element in them
//     ResNet-50's, a kernel in 0.4 kept, bf16 gradients, 8-bit states   34 us: 2.8 TB/s of traffic, instructions
//         (70 % of the issue slots) and the latency of the chain
template <int BITS, int N, bool MASKED>
__global__ void __launch_bounds__(kThreads, MASKED ? 6 : 5) adamw_kernel(const Chunk* __restrict__ chunks, uint32_t begin, uint32_t t0,
                                                            Grads<N> grads, AdamArgs a) {
    __shared__ uint8_t lists[MASKED ? kThreads / 32 : 1][kBlock];
    const Chunk t = chunks[begin + blockIdx.x];
    const void* gp = grads.at[t.tensor - t0];
    if (!gp) return;                               // a tensor without a gradient is left alone
    const bool wide = wide_grad(gp, t.grad_dtype) && (reinterpret_cast<uintptr_t>(t.param) & 31) == 0;
    gp = static_cast<const char*>(gp) + t.first * (t.grad_dtype == PP_F32 ? 4 : 2);
    const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
    const float shrink = fmaf(-a.lr, t.decay, 1.0f);
    const uint32_t le = threadIdx.x * 8, warp = le & ~(kBlock - 1);
    if (warp >= t.count) return;                   // whole warps
    if constexpr (!MASKED) {
        if (wide && warp + kBlock <= t.count) {
            if (t.grad_dtype == PP_F32)
                dense_block<BITS, PP_F32>(t, gp, le, gs, shrink, a);
            else if (t.grad_dtype == PP_F16)
                dense_block<BITS, PP_F16>(t, gp, le, gs, shrink, a);
            else
                dense_block<BITS, PP_BF16>(t, gp, le, gs, shrink, a);
            return;
        }
    }
    const uint32_t keep = kept8(t.taps, t.tap, t.count, le, in_chunk(t.count, le));
    if constexpr (MASKED) {
        uint8_t* list = lists[threadIdx.x / 32];
        const int count = list_kept(keep, list);
        __syncwarp();
        if (count <= 128) {
            if (!count) return;                    // its states are zero and stay so
            Listed<BITS, 4> x;
            x.load(t, gp, warp, list, count, a);
            x.step(t, warp, count, gs, shrink, a);
            return;
        }
    }
    any_block<BITS>(t, gp, le, keep, gs, shrink, a);
}

template <int N>
Grads<N> take(const void* const* grads, int first, int count) {
    Grads<N> g;
    for (int i = 0; i < N; ++i) g.at[i] = i < count ? grads[first + i] : nullptr;
    return g;
}

bool known(int dtype) { return dtype == PP_F32 || dtype == PP_F16 || dtype == PP_BF16; }

int check_grads(const pp_tensors* h, const void* const* grads) {
    if (!h) return PP_ERR_NULL;
    if (!h->tensors.empty() && !grads) return PP_ERR_NULL;
    if (!h->dev) return PP_ERR_NOT_BOUND;
    for (size_t i = 0; i < h->tensors.size(); ++i)
        if (reinterpret_cast<uintptr_t>(grads[i]) % (h->tensors[i].grad_dtype == PP_F32 ? 4 : 2)) return PP_ERR_ALIGN;
    return PP_OK;
}

// whether two of the stretches of memory that a step writes share a byte: their elements would be written in no order
bool shared(int n, const int64_t* numel, float* const* params, void* const* copies) {
    std::vector<std::pair<uintptr_t, uintptr_t>> at;      // begin, end
    for (int i = 0; i < n; ++i) {
        const uintptr_t p = params && params[i] ? reinterpret_cast<uintptr_t>(params[i]) : 0;
        const uintptr_t c = copies && copies[i] ? reinterpret_cast<uintptr_t>(copies[i]) : 0;
        if (p && numel[i]) at.emplace_back(p, p + (uintptr_t)numel[i] * 4);
        if (c && numel[i]) at.emplace_back(c, c + (uintptr_t)numel[i] * 2);
    }
    std::sort(at.begin(), at.end());
    for (size_t i = 1; i < at.size(); ++i)
        if (at[i].first < at[i - 1].second) return true;
    return false;
}

int launched() { return cudaGetLastError() == cudaSuccess ? PP_OK : PP_ERR_CUDA; }

}  // namespace

extern "C" {

int pp_tensors_create(int n, const int64_t* numel, const int* grad_dtypes, const uint16_t* const* taps,
                      float* const* params, void* const* copies, int copy_dtype, const float* decay,
                      pp_tensors_handle* out) {
    if (n < 0 || n > (1 << 20)) return PP_ERR_SHAPE;
    if (!out || (n && (!numel || !grad_dtypes))) return PP_ERR_NULL;
    if (copies && copy_dtype != PP_F16 && copy_dtype != PP_BF16) return PP_ERR_DTYPE;
    for (int i = 0; i < n; ++i) {
        if (numel[i] < 0 || numel[i] > kMaxNumel) return PP_ERR_SHAPE;
        if (!known(grad_dtypes[i])) return PP_ERR_DTYPE;
        if (taps && taps[i] && numel[i] % 9) return PP_ERR_SHAPE;
        if (taps && reinterpret_cast<uintptr_t>(taps[i]) % 2) return PP_ERR_ALIGN;
        if (params && numel[i] && !params[i]) return PP_ERR_NULL;
        if (params && reinterpret_cast<uintptr_t>(params[i]) % 4) return PP_ERR_ALIGN;
        if (copies && reinterpret_cast<uintptr_t>(copies[i]) % 2) return PP_ERR_ALIGN;
        if (decay && !std::isfinite(decay[i])) return PP_ERR_ARG;
    }
    try {
        if (shared(n, numel, params, copies)) return PP_ERR_BUFFER;
        pp_tensors* h = new pp_tensors;
        struct Guard {
            pp_tensors* h;
            ~Guard() { delete h; }
        } guard{h};
        uint64_t chunks = 0, spans = 0;
        for (int i = 0; i < n; ++i) {
            const Tensor t{numel[i], h->state_elements, grad_dtypes[i], taps && taps[i]};
            h->tensors.push_back(t);
            h->first_chunk.push_back((uint32_t)chunks);
            h->state_elements += (numel[i] + kBlock - 1) / kBlock * kBlock;
            h->first_span.push_back((uint32_t)spans);
            if (params) chunks += (uint64_t)((numel[i] + kChunk - 1) / kChunk);      // the norm reads spans alone
            spans += (uint64_t)((numel[i] + kSpan - 1) / kSpan);
            if (std::max(chunks, spans) > 0x7FFFFFFFu) return PP_ERR_SHAPE;
        }
        h->first_chunk.push_back((uint32_t)chunks);
        h->first_span.push_back((uint32_t)spans);
        h->copy_dtype = copy_dtype;
        h->has_params = params != nullptr;
        h->off_spans = (chunks * sizeof(Chunk) + 255) / 256 * 256;
        h->off_sums = (h->off_spans + spans * sizeof(Span) + 255) / 256 * 256;
        const size_t launches = ((size_t)n + kMaxGrads - 1) / kMaxGrads;
        h->image.assign(h->off_sums + kCounterBytes + std::max<size_t>(1, launches) * kSumCtas * sizeof(double), 0);
        Chunk* c = reinterpret_cast<Chunk*>(h->image.data());
        const Chunk* const first = c;
        for (int i = 0; params && i < n; i += kMaxGrads) {
            const int end = std::min(n, i + kMaxGrads);
            for (const bool masked : {true, false}) {
                for (int k = i; k < end; ++k) {
                    const Tensor& t = h->tensors[k];
                    if (t.masked != masked) continue;
                    for (int64_t e = 0; e < t.numel; e += kChunk, ++c) {
                        c->param = params[k] + e;
                        c->copy = copies && copies[k] ? static_cast<uint16_t*>(copies[k]) + e : nullptr;
                        c->taps = masked ? taps[k] + e / 9 : nullptr;
                        c->state = t.state + e;
                        c->first = e;
                        c->tensor = (uint32_t)k;
                        c->count = (uint16_t)std::min<int64_t>(kChunk, t.numel - e);
                        c->tap = (uint8_t)(e % 9);
                        c->grad_dtype = (uint8_t)t.grad_dtype;
                        c->decay = decay ? decay[k] : 0.0f;
                    }
                }
                if (masked) h->masked_end.push_back((uint32_t)(c - first));
            }
        }
        Span* sp = reinterpret_cast<Span*>(h->image.data() + h->off_spans);
        for (int k = 0; k < n; ++k) {
            const Tensor& t = h->tensors[k];
            for (int64_t e = 0; e < t.numel; e += kSpan)
                *sp++ = {t.masked ? taps[k] + e / 9 : nullptr, e, (uint32_t)k, (uint32_t)std::min<int64_t>(kSpan, t.numel - e),
                         (uint32_t)(e % 9), (uint32_t)t.grad_dtype};
        }
        guard.h = nullptr;
        *out = h;
        return PP_OK;
    } catch (const std::bad_alloc&) {
        return PP_ERR_ALLOC;
    }
}

int pp_tensors_query(pp_tensors_handle h, int key, int64_t* value) {
    if (!h || !value) return PP_ERR_NULL;
    switch (key) {
        case PP_TQ_COUNT: *value = (int64_t)h->tensors.size(); return PP_OK;
        case PP_TQ_TABLE_BYTES: *value = (int64_t)h->image.size(); return PP_OK;
        case PP_TQ_STATE_ELEMENTS: *value = h->state_elements; return PP_OK;
    }
    if (key >= PP_TQ_STATE_OFFSET && (size_t)(key - PP_TQ_STATE_OFFSET) < h->tensors.size()) {
        *value = h->tensors[key - PP_TQ_STATE_OFFSET].state;
        return PP_OK;
    }
    return PP_ERR_ARG;
}

int pp_tensors_bind(pp_tensors_handle h, void* dev, size_t bytes, void* stream) {
    if (!h || !dev) return PP_ERR_NULL;
    if (bytes < h->image.size()) return PP_ERR_BUFFER;
    if (reinterpret_cast<uintptr_t>(dev) % 256) return PP_ERR_ALIGN;
    if (cudaMemcpyAsync(dev, h->image.data(), h->image.size(), cudaMemcpyHostToDevice,
                        static_cast<cudaStream_t>(stream)) != cudaSuccess) {
        cudaGetLastError();
        return PP_ERR_CUDA;
    }
    h->dev = static_cast<unsigned char*>(dev);
    return PP_OK;
}

int pp_tensors_destroy(pp_tensors_handle h) {
    delete h;
    return PP_OK;
}

int pp_grad_norm(pp_tensors_handle h, const void* const* grads, double max_norm, float* out, void* stream) {
    if (const int e = check_grads(h, grads)) return e;
    if (!out) return PP_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(out) % 4) return PP_ERR_ALIGN;
    if (!(max_norm > 0)) return PP_ERR_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Span* spans = reinterpret_cast<const Span*>(h->dev + h->off_spans);
    unsigned* counter = reinterpret_cast<unsigned*>(h->dev + h->off_sums);
    double* sums = reinterpret_cast<double*>(h->dev + h->off_sums + kCounterBytes);
    const int n = (int)h->tensors.size();
    // A call leaves its counters at zero, but one of several launches that failed between them has not: such a
    // handle's calls begin with zeros of their own.
    if (n > kMaxGrads && cudaMemsetAsync(counter, 0, kCounterBytes, st) != cudaSuccess) {
        cudaGetLastError();
        return PP_ERR_CUDA;
    }
    unsigned all = 0;
    for (int pass = 0; pass < 2; ++pass) {        // count the partial sums, then launch
        unsigned done = 0;
        int i = 0;
        do {
            const int count = std::min(n - i, kMaxGrads);
            const uint32_t begin = h->first_span[i], end = h->first_span[i + count];
            const bool wide = std::any_of(h->tensors.begin() + i, h->tensors.begin() + i + count,
                                          [](const Tensor& t) { return t.grad_dtype == PP_F32; });
            const unsigned grid = std::max(1u, std::min<uint32_t>(end - begin, kSMs * (wide ? 5 : 4)));
            if (pass) {
                const auto launch = [&](auto many, auto with_wide) {
                    constexpr int M = decltype(many)::value;
                    grad_norm_kernel<M, decltype(with_wide)::value><<<grid, kThreads, 0, st>>>(
                        spans, begin, end, (uint32_t)i, take<M>(grads, i, count), sums, counter, done, all, (float)max_norm, out);
                };
                using Few = std::integral_constant<int, kFewGrads>;
                using Many = std::integral_constant<int, kMaxGrads>;
                if (count <= kFewGrads)
                    wide ? launch(Few(), std::true_type()) : launch(Few(), std::false_type());
                else
                    wide ? launch(Many(), std::true_type()) : launch(Many(), std::false_type());
                if (const int e = launched()) return e;
            }
            done += grid;
            i += count;
        } while (i < n);
        all = done;
    }
    return PP_OK;
}

int pp_adamw_step(pp_tensors_handle h, const void* const* grads, int state_bits, void* m, void* v, float* m_scale,
                  float* v_scale, double lr, double beta1, double beta2, double eps, int64_t step, uint32_t seed,
                  const float* grad_scale, void* stream) {
    if (const int e = check_grads(h, grads)) return e;
    if (!h->has_params) return PP_ERR_NOT_BOUND;
    if (state_bits != 32 && state_bits != 8) return PP_ERR_ARG;
    if (!std::isfinite(lr) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) || !(eps >= 0) ||
        !std::isfinite(eps) || step < 1)
        return PP_ERR_ARG;
    const uint32_t all = h->first_chunk.back();
    if (!all) return PP_OK;
    if (!m || !v || (state_bits == 8 && (!m_scale || !v_scale))) return PP_ERR_NULL;
    const auto off = [](const void* p, size_t k) { return reinterpret_cast<uintptr_t>(p) % k != 0; };
    if (off(m, 32) || off(v, 32) || off(m_scale, 4) || off(v_scale, 4) || off(grad_scale, 4)) return PP_ERR_ALIGN;
    AdamArgs a{};
    a.lr = (float)lr;
    a.one = 1.0f;
    a.step_size = (float)(lr / (1 - std::pow(beta1, (double)step)));
    a.b1 = (float)beta1;
    a.b2 = (float)beta2;
    a.c1 = (float)(1 - beta1);
    a.c2 = (float)(1 - beta2);
    a.inv_bc2 = (float)(1 / (1 - std::pow(beta2, (double)step)));
    a.eps = (float)eps;
    a.key = mix(seed + (uint32_t)step * 0x9E3779B1u);
    a.copy_dtype = h->copy_dtype;
    a.grad_scale = grad_scale;
    a.m = m;
    a.v = v;
    a.m_scale = m_scale;
    a.v_scale = v_scale;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Chunk* chunks = reinterpret_cast<const Chunk*>(h->dev);
    const int n = (int)h->tensors.size();
    for (int i = 0; i < n; i += kMaxGrads) {
        const int count = std::min(n - i, kMaxGrads);
        // chunks of tensors with masks, then those without: by one kernel where these are few, or all are at
        // work at once
        const uint32_t begin = h->first_chunk[i], end = h->first_chunk[i + count], masked = h->masked_end[i / kMaxGrads];
        const bool one = masked > begin && ((end - masked) * 32 <= end - begin || end - begin <= kSMs * 5);
        const uint32_t split = one ? end : masked;
        const bool few = count <= kFewGrads;
        const auto launch = [&](auto bits, auto many, auto with_mask, uint32_t from, uint32_t to) {
            constexpr int B = decltype(bits)::value, M = decltype(many)::value;
            if (from == to) return PP_OK;
            adamw_kernel<B, M, decltype(with_mask)::value><<<to - from, kThreads, 0, st>>>(
                chunks, from, (uint32_t)i, take<M>(grads, i, count), a);
            return (pp_status)launched();
        };
        const auto both = [&](auto bits, auto many) {
            const int e = launch(bits, many, std::true_type(), begin, split);
            return e ? e : (int)launch(bits, many, std::false_type(), split, end);
        };
        using Few = std::integral_constant<int, kFewGrads>;
        using Many = std::integral_constant<int, kMaxGrads>;
        using Eight = std::integral_constant<int, 8>;
        using Full = std::integral_constant<int, 32>;
        const int e = state_bits == 8 ? (few ? both(Eight(), Few()) : both(Eight(), Many()))
                                      : (few ? both(Full(), Few()) : both(Full(), Many()));
        if (e) return e;
    }
    return PP_OK;
}

}  // extern "C"
