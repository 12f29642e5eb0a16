// Group norm with its activation on channels-last activations, forward and backward, for masked
// retraining.
//
// x is [N][pixels][C] with C innermost.  For every sample and group of C / G channels, over its
// M = pixels C / G values,
//     mean = sum x / M,  var = sum (x - mean)^2 / M,  rstd = 1 / sqrt(var + eps),
//     xh = (x - mean) rstd,  z = gamma xh + beta,  y = act(z);
// backward, with dz = dy act'(z),
//     dbeta_c = sum over samples and pixels of dz,  dgamma_c = sum of dz xh,
//     dx = rstd (gamma dz - A / M - xh B / M),  A = sum over the group of gamma dz,  B = of gamma dz xh.
//
// What bounds it is memory: a forward pass must read x and write y, a backward pass read x and dy and
// write dx, for 10 to 30 operations an element.
//
// Streamed form: one kernel sums (a CTA takes a stretch of pixels of a sample, a thread always the same
// V channels, so that a warp reads whole rows), one joins a sample's parts, one applies.  The second
// reading comes from L2 where a call's tensors fit there.
//
// Means and squares are joined pairwise as (count, mean, sum of squared distances from the mean): a
// plain sum of squares would lose the variance of values far from zero.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "patconv.h"

namespace {

constexpr int kThreads = 256;

// -------------------------------------------------------------------------------- vectors of values

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T v[V];
};

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__half x) { return __half2float(x); }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void narrow(float x, float& y) { y = x; }
__device__ __forceinline__ void narrow(float x, __half& y) { y = __float2half_rn(x); }
__device__ __forceinline__ void narrow(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load(const T* p) {
    return *reinterpret_cast<const Vec<T, V>*>(p);
}
template <typename T, int V>
__device__ __forceinline__ void store(T* p, const Vec<T, V>& v) {
    *reinterpret_cast<Vec<T, V>*>(p) = v;
}

// -------------------------------------------------------------------------------- joining moments

struct Moments {
    float n, mean, m2;
};
__device__ __forceinline__ Moments join(const Moments& a, const Moments& b) {
    const float n = a.n + b.n;
    if (n == 0.0f) return a;
    const float f = b.n / n, d = b.mean - a.mean;
    return {n, fmaf(d, f, a.mean), a.m2 + fmaf(d * d, a.n * f, b.m2)};
}
__device__ __forceinline__ Moments join_warp(Moments m) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const Moments b{__shfl_down_sync(0xffffffffu, m.n, o), __shfl_down_sync(0xffffffffu, m.mean, o),
                        __shfl_down_sync(0xffffffffu, m.m2, o)};
        m = join(m, b);
    }
    return m;
}
__device__ __forceinline__ float sum_warp(float s) {
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_down_sync(0xffffffffu, s, o);
    return s;
}

// -------------------------------------------------------------------------------- activations

__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }
__device__ __forceinline__ float activated(float z, int act) {
    if (act == PP_ACT_RELU) return z > 0.0f ? z : z != z ? z : 0.0f;
    if (act == PP_ACT_SILU) return __fdividef(z, 1.0f + __expf(-z));
    return z;
}
// act'(z)
__device__ __forceinline__ float slope(float z, int act) {
    if (act == PP_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (act == PP_ACT_SILU) {
        const float s = sigmoid(z);
        return fmaf(z * s, 1.0f - s, s);
    }
    return 1.0f;
}

// -------------------------------------------------------------------------------- streamed kernels

struct NormArgs {
    const void *x, *dy;
    int64_t x_pixel, x_sample, dy_pixel, dy_sample;   // strides in elements
    const float *gamma, *beta;
    const float *mean, *rstd;         // [N][G]
    float *mean_out, *rstd_out;
    void* out;                        // y or dx: dense
    float *dgamma, *dbeta;
    float* parts;                     // of a pass's sums
    float* sums;                      // backward: [N][2][C] sums over a sample, then [N][G][2] A / M, B / M
    int64_t pixels;
    int N, C, G, cpg, act;
    int cols, rows;                   // vectors of a row a CTA covers, rows it covers at a time
    int tiles;                        // CTAs side by side cover a row
    int chunk, chunks;                // pixels of a CTA, CTAs down a sample
    float eps;
};

// Where a thread stands: its column (V channels from c), its first row, its CTA's pixels.
template <int V>
struct Place {
    int c, row, n;
    int64_t begin, end;
    bool on;
    __device__ Place(const NormArgs& a) {
        const int tile = blockIdx.y;
        const int col = threadIdx.x % a.cols;
        row = threadIdx.x / a.cols;
        c = (tile * a.cols + col) * V;
        on = row < a.rows && c < a.C;
        n = blockIdx.z;
        begin = (int64_t)blockIdx.x * a.chunk;
        end = min(begin + a.chunk, a.pixels);
    }
};

// Sums of a stretch of pixels, a channel at a time: parts[n][chunk][c] = (mean, m2); the count is the
// stretch's length.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) norm_moments(NormArgs a) {
    constexpr int U = V >= 4 ? 4 : 8;
    __shared__ float s_mean[kThreads * V], s_m2[kThreads * V], s_n[kThreads];
    const Place<V> at(a);
    float n = 0.0f, mean[V] = {}, m2[V] = {};
    if (at.on) {
        const T* x = static_cast<const T*>(a.x) + at.n * a.x_sample + at.c;
        for (int64_t p = at.begin + at.row; p < at.end; p += U * a.rows) {
            Vec<T, V> v[U];
            int k = 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * a.rows < at.end) {
                    v[u] = load<T, V>(x + (p + u * a.rows) * a.x_pixel);
                    k = u + 1;
                }
            // a batch's values by their distance from its first one: a constant's mean and variance are
            // exact, and the sum of squares is at most k + 1 times what is left of it
            const float inv = __fdividef(1.0f, (float)k), total = n + k, f = __fdividef((float)k, total), w = n * f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float x0 = widen(v[0].v[i]);
                float s = 0.0f, q = 0.0f;
#pragma unroll
                for (int u = 1; u < U; ++u) {
                    const float d = u < k ? widen(v[u].v[i]) - x0 : 0.0f;
                    s += d;
                    q = fmaf(d, d, q);
                }
                q = fmaf(-s * inv, s, q);
                const float d = fmaf(s, inv, x0) - mean[i];
                mean[i] = fmaf(d, f, mean[i]);
                m2[i] += fmaf(d * d, w, q < 0.0f ? 0.0f : q);
            }
            n = total;
        }
    }
    s_n[threadIdx.x] = n;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        s_mean[i * kThreads + threadIdx.x] = mean[i];
        s_m2[i * kThreads + threadIdx.x] = m2[i];
    }
    __syncthreads();
    for (int j = threadIdx.x; j < a.cols * V; j += kThreads) {       // a channel of the tile each
        const int col = j / V, i = j % V, c = blockIdx.y * a.cols * V + j;
        if (c >= a.C) break;
        Moments m{0.0f, 0.0f, 0.0f};
        for (int r = 0; r < a.rows; ++r) {
            const int t = r * a.cols + col;
            m = join(m, {s_n[t], s_mean[i * kThreads + t], s_m2[i * kThreads + t]});
        }
        float* out = a.parts + (((int64_t)at.n * a.chunks + blockIdx.x) * a.C + c) * 2;
        out[0] = m.mean;
        out[1] = m.m2;
    }
}

// A group's mean and rstd from its channels' parts: a warp a group.
__global__ void __launch_bounds__(kThreads) norm_join(NormArgs a) {
    const int64_t g = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (g >= (int64_t)a.N * a.G) return;
    const int n = (int)(g / a.G), c0 = (int)(g % a.G) * a.cpg, lane = threadIdx.x % 32;
    Moments m{0.0f, 0.0f, 0.0f};
    for (int64_t j = lane; j < (int64_t)a.chunks * a.cpg; j += 32) {
        const int k = (int)(j / a.cpg), c = c0 + (int)(j % a.cpg);
        const float* p = a.parts + (((int64_t)n * a.chunks + k) * a.C + c) * 2;
        m = join(m, {(float)min((int64_t)a.chunk, a.pixels - (int64_t)k * a.chunk), p[0], p[1]});
    }
    m = join_warp(m);
    if (lane == 0) {
        const float var = m.m2 / ((float)a.pixels * a.cpg);
        a.mean_out[g] = m.mean;
        a.rstd_out[g] = 1.0f / sqrtf(var + a.eps);
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(kThreads) norm_apply(NormArgs a) {
    constexpr int U = 4;
    const Place<V> at(a);
    if (!at.on) return;
    float mean[V], scale[V], shift[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = at.c + i, g = at.n * a.G + c / a.cpg;
        mean[i] = a.mean[g];
        scale[i] = a.rstd[g] * (a.gamma ? a.gamma[c] : 1.0f);
        shift[i] = a.beta ? a.beta[c] : 0.0f;
    }
    const T* x = static_cast<const T*>(a.x) + at.n * a.x_sample + at.c;
    T* y = static_cast<T*>(a.out) + (int64_t)at.n * a.pixels * a.C + at.c;
    for (int64_t p = at.begin + at.row; p < at.end; p += U * a.rows) {
        Vec<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u * a.rows < at.end) v[u] = load<T, V>(x + (p + u * a.rows) * a.x_pixel);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * a.rows >= at.end) break;
#pragma unroll
            for (int i = 0; i < V; ++i)
                narrow(activated(fmaf(widen(v[u].v[i]) - mean[i], scale[i], shift[i]), a.act), v[u].v[i]);
            store<T, V>(y + (p + u * a.rows) * a.C, v[u]);
        }
    }
}

// -------------------------------------------------------------------------------- backward

template <int V>
struct Affine {                       // of a thread's channels
    float mean[V], rstd[V], gamma[V], beta[V];
    __device__ Affine(const NormArgs& a, int n, int c0) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = c0 + i, g = n * a.G + c / a.cpg;
            mean[i] = a.mean[g];
            rstd[i] = a.rstd[g];
            gamma[i] = a.gamma ? a.gamma[c] : 1.0f;
            beta[i] = a.beta ? a.beta[c] : 0.0f;
        }
    }
};

// parts[n][chunk][c] = (sum of dz, sum of dz xh) over the stretch
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) norm_back_sums(NormArgs a) {
    constexpr int U = 2;
    __shared__ float s_b[kThreads * V], s_g[kThreads * V];
    const Place<V> at(a);
    float sb[V] = {}, sg[V] = {};
    if (at.on) {
        const Affine<V> f(a, at.n, at.c);
        const T* x = static_cast<const T*>(a.x) + at.n * a.x_sample + at.c;
        const T* dy = static_cast<const T*>(a.dy) + at.n * a.dy_sample + at.c;
        for (int64_t p = at.begin + at.row; p < at.end; p += U * a.rows) {
            Vec<T, V> v[U], w[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * a.rows < at.end) {
                    v[u] = load<T, V>(x + (p + u * a.rows) * a.x_pixel);
                    w[u] = load<T, V>(dy + (p + u * a.rows) * a.dy_pixel);
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (p + u * a.rows >= at.end) break;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xh = (widen(v[u].v[i]) - f.mean[i]) * f.rstd[i];
                    const float dz = widen(w[u].v[i]) * slope(fmaf(xh, f.gamma[i], f.beta[i]), a.act);
                    sb[i] += dz;
                    sg[i] = fmaf(dz, xh, sg[i]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        s_b[i * kThreads + threadIdx.x] = sb[i];
        s_g[i * kThreads + threadIdx.x] = sg[i];
    }
    __syncthreads();
    for (int j = threadIdx.x; j < a.cols * V; j += kThreads) {
        const int col = j / V, i = j % V, c = blockIdx.y * a.cols * V + j;
        if (c >= a.C) break;
        float b = 0.0f, g = 0.0f;
        for (int r = 0; r < a.rows; ++r) {
            b += s_b[i * kThreads + r * a.cols + col];
            g += s_g[i * kThreads + r * a.cols + col];
        }
        float* out = a.parts + (((int64_t)at.n * a.chunks + blockIdx.x) * a.C + c) * 2;
        out[0] = b;
        out[1] = g;
    }
}

// Over a sample's stretches: sums[n][c] = (dz, dz xh) and, a CTA a group, A / M and B / M.
__global__ void __launch_bounds__(kThreads) norm_back_join(NormArgs a) {
    __shared__ float s_a[kThreads / 32], s_b[kThreads / 32];
    const int n = blockIdx.y, g = blockIdx.x;
    float A = 0.0f, B = 0.0f;
    for (int j = threadIdx.x; j < a.cpg; j += kThreads) {
        const int c = g * a.cpg + j;
        float b = 0.0f, s = 0.0f;
        const float* p = a.parts + ((int64_t)n * a.chunks * a.C + c) * 2;
        for (int k = 0; k < a.chunks; ++k, p += 2 * (int64_t)a.C) {
            b += p[0];
            s += p[1];
        }
        float* out = a.sums + ((int64_t)n * a.C + c) * 2;
        out[0] = b;
        out[1] = s;
        const float gamma = a.gamma ? a.gamma[c] : 1.0f;
        A = fmaf(gamma, b, A);
        B = fmaf(gamma, s, B);
    }
    A = sum_warp(A);
    B = sum_warp(B);
    if (threadIdx.x % 32 == 0) {
        s_a[threadIdx.x / 32] = A;
        s_b[threadIdx.x / 32] = B;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 32; ++w) {
            A += s_a[w];
            B += s_b[w];
        }
        const float inv = 1.0f / ((float)a.pixels * a.cpg);
        float* out = a.sums + (int64_t)a.N * a.C * 2 + ((int64_t)n * a.G + g) * 2;
        out[0] = A * inv;
        out[1] = B * inv;
    }
}

// dx, and in the CTAs of the last blockIdx.z the sums over the samples
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) norm_back_apply(NormArgs a) {
    constexpr int U = 2;
    if (blockIdx.z == a.N) {
        const int64_t c = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kThreads + threadIdx.x;
        for (int64_t j = c; j < a.C; j += (int64_t)gridDim.x * gridDim.y * kThreads) {
            float b = 0.0f, g = 0.0f;
            for (int n = 0; n < a.N; ++n) {
                b += a.sums[((int64_t)n * a.C + j) * 2];
                g += a.sums[((int64_t)n * a.C + j) * 2 + 1];
            }
            if (a.dbeta) a.dbeta[j] = b;
            if (a.dgamma) a.dgamma[j] = g;
        }
        return;
    }
    const Place<V> at(a);
    if (!at.on) return;
    const Affine<V> f(a, at.n, at.c);
    float A[V], B[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float* s = a.sums + (int64_t)a.N * a.C * 2 + ((int64_t)at.n * a.G + (at.c + i) / a.cpg) * 2;
        A[i] = s[0];
        B[i] = s[1];
    }
    const T* x = static_cast<const T*>(a.x) + at.n * a.x_sample + at.c;
    const T* dy = static_cast<const T*>(a.dy) + at.n * a.dy_sample + at.c;
    T* dx = static_cast<T*>(a.out) + (int64_t)at.n * a.pixels * a.C + at.c;
    for (int64_t p = at.begin + at.row; p < at.end; p += U * a.rows) {
        Vec<T, V> v[U], w[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u * a.rows < at.end) {
                v[u] = load<T, V>(x + (p + u * a.rows) * a.x_pixel);
                w[u] = load<T, V>(dy + (p + u * a.rows) * a.dy_pixel);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * a.rows >= at.end) break;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (widen(v[u].v[i]) - f.mean[i]) * f.rstd[i];
                const float dz = widen(w[u].v[i]) * slope(fmaf(xh, f.gamma[i], f.beta[i]), a.act);
                // the product is rounded by itself, so that dx of a group of one value is zero
                narrow(f.rstd[i] * fmaf(-xh, B[i], __fmul_rn(f.gamma[i], dz) - A[i]), v[u].v[i]);
            }
            store<T, V>(dx + (p + u * a.rows) * a.C, v[u]);
        }
    }
}

// -------------------------------------------------------------------------------- host

struct Shape {
    int dtype, N, C, G;
    int64_t pixels;
};

size_t size_of(int dtype) { return dtype == PP_F32 ? 4 : 2; }

int check_shape(const Shape& s) {
    if (s.dtype != PP_F32 && s.dtype != PP_F16 && s.dtype != PP_BF16) return PP_ERR_DTYPE;
    if (s.N < 0 || s.N > 65534 || s.C < 1 || s.C > (1 << 20) || s.G < 1 || s.C % s.G || s.pixels < 0 ||
        s.pixels > INT_MAX)
        return PP_ERR_SHAPE;
    if (s.N && s.pixels && s.pixels > (int64_t(1) << 42) / s.N / s.C) return PP_ERR_SHAPE;
    return PP_OK;
}

struct Split {
    int V, cols, rows, tiles, chunk, chunks;
};

// V channels a thread (16 bytes where `align`, the common alignment of addresses and strides in bytes,
// allows it), a row's vectors over the threads of one or more CTAs, and stretches of pixels such that
// there are a few CTAs for every SM but no CTA has less than 16 KB.
Split split_of(const Shape& s, int align) {
    Split p;
    p.V = std::max<int>(1, std::min(align, 16) / (int)size_of(s.dtype));
    const int vectors = s.C / p.V;
    p.tiles = (vectors + kThreads - 1) / kThreads;
    p.cols = (vectors + p.tiles - 1) / p.tiles;
    p.rows = kThreads / p.cols;
    const int64_t row = (int64_t)p.cols * p.V * size_of(s.dtype);
    const int64_t least = std::max<int64_t>((16384 + row - 1) / row, p.rows);
    const int64_t want = std::max<int64_t>(1, (152 * 8 + (int64_t)s.N * p.tiles - 1) / ((int64_t)s.N * p.tiles));
    p.chunk = (int)std::max(least, (s.pixels + want - 1) / want);
    p.chunks = (int)((s.pixels + p.chunk - 1) / p.chunk);
    return p;
}

// floats of the workspace: a part a channel and stretch (with the most stretches any alignment gives),
// then mean and rstd, or the backward pass's sums
struct Space {
    size_t parts, stats, sums;
    size_t bytes() const { return (parts + stats + sums) * sizeof(float); }
};
Space space_of(const Shape& s, bool backward) {
    int chunks = 0;
    for (int align = (int)size_of(s.dtype); align <= 16; align *= 2)
        if ((int64_t)s.C * size_of(s.dtype) % align == 0) chunks = std::max(chunks, split_of(s, align).chunks);
    Space w{(size_t)s.N * chunks * s.C * 2, 0, 0};
    if (backward)
        w.sums = (size_t)s.N * s.C * 2 + (size_t)s.N * s.G * 2;
    else
        w.stats = (size_t)s.N * s.G * 2;
    return w;
}

int align_of(const void* p) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p) | 16;
    return (int)(a & -a);
}
int align_of(int64_t elements, int dtype) {
    const uint64_t a = (uint64_t)elements * size_of(dtype) | 16;
    return (int)(a & -a);
}

// strides of an input: pixels may lie further apart than C (channels of a wider tensor)
int check_input(const Shape& s, const void* p, int64_t pixel, int64_t sample) {
    if (!p) return PP_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(p) % size_of(s.dtype)) return PP_ERR_ALIGN;
    if (s.pixels > 1 && (pixel < s.C || pixel > (int64_t(1) << 31))) return PP_ERR_SHAPE;
    if (s.N > 1 && (sample < 0 || sample > (int64_t(1) << 42))) return PP_ERR_SHAPE;
    return PP_OK;
}

// bytes from an input's first element to the end of its last
size_t extent(const Shape& s, int64_t pixel, int64_t sample) {
    return (size_t)((s.N - 1) * sample + (s.pixels - 1) * pixel + s.C) * size_of(s.dtype);
}
bool overlap(const void* p, size_t pn, const void* q, size_t qn) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a < b + qn && b < a + pn;
}

template <typename T>
cudaError_t forward(const NormArgs& a, int V, cudaStream_t st) {
    const dim3 grid(a.chunks, a.tiles, a.N);
    const unsigned joins = (unsigned)(((int64_t)a.N * a.G + kThreads / 32 - 1) / (kThreads / 32));
#define PP_RUN(VV)                                                \
    case VV:                                                      \
        norm_moments<T, VV><<<grid, kThreads, 0, st>>>(a);        \
        norm_join<<<joins, kThreads, 0, st>>>(a);                 \
        norm_apply<T, VV><<<grid, kThreads, 0, st>>>(a);          \
        break;
    switch (V) {
        PP_RUN(1)
        PP_RUN(2)
        PP_RUN(4)
        case 8:
            if constexpr (sizeof(T) == 2) {
                norm_moments<T, 8><<<grid, kThreads, 0, st>>>(a);
                norm_join<<<joins, kThreads, 0, st>>>(a);
                norm_apply<T, 8><<<grid, kThreads, 0, st>>>(a);
            }
            break;
    }
#undef PP_RUN
    return cudaGetLastError();
}

template <typename T>
cudaError_t backward(const NormArgs& a, int V, cudaStream_t st) {
    const dim3 grid(a.chunks, a.tiles, a.N), last(a.chunks, a.tiles, a.N + 1), join(a.G, a.N);
#define PP_RUN(VV)                                                \
    case VV:                                                      \
        norm_back_sums<T, VV><<<grid, kThreads, 0, st>>>(a);      \
        norm_back_join<<<join, kThreads, 0, st>>>(a);             \
        norm_back_apply<T, VV><<<last, kThreads, 0, st>>>(a);     \
        break;
    switch (V) {
        PP_RUN(1)
        PP_RUN(2)
        PP_RUN(4)
        case 8:
            if constexpr (sizeof(T) == 2) {
                norm_back_sums<T, 8><<<grid, kThreads, 0, st>>>(a);
                norm_back_join<<<join, kThreads, 0, st>>>(a);
                norm_back_apply<T, 8><<<last, kThreads, 0, st>>>(a);
            }
            break;
    }
#undef PP_RUN
    return cudaGetLastError();
}

void take(NormArgs& a, const Shape& s, const Split& p) {
    a.N = s.N;
    a.C = s.C;
    a.G = s.G;
    a.cpg = s.C / s.G;
    a.pixels = s.pixels;
    a.cols = p.cols;
    a.rows = p.rows;
    a.tiles = p.tiles;
    a.chunk = p.chunk;
    a.chunks = p.chunks;
}

bool off4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; }

}  // namespace

extern "C" {

int pp_group_norm_workspace_size(int dtype, int N, int64_t pixels, int C, int G, int backward, size_t* bytes) {
    if (!bytes) return PP_ERR_NULL;
    const Shape s{dtype, N, C, G, pixels};
    if (const int e = check_shape(s)) return e;
    if (backward != 0 && backward != 1) return PP_ERR_ARG;
    *bytes = N && pixels ? space_of(s, backward).bytes() : 0;
    return PP_OK;
}

int pp_group_norm(const void* x, int64_t x_pixel, int64_t x_sample, int dtype, int N, int64_t pixels, int C, int G,
                  const float* gamma, const float* beta, float eps, int act, void* y, float* mean, float* rstd,
                  void* workspace, size_t workspace_bytes, void* stream) {
    const Shape s{dtype, N, C, G, pixels};
    if (const int e = check_shape(s)) return e;
    if (act != PP_ACT_NONE && act != PP_ACT_RELU && act != PP_ACT_SILU) return PP_ERR_ARG;
    if (!(eps >= 0) || !std::isfinite(eps)) return PP_ERR_ARG;
    if (!N || !pixels) return PP_OK;
    if (const int e = check_input(s, x, x_pixel, x_sample)) return e;
    if (!y || !workspace) return PP_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(y) % size_of(dtype) || off4(gamma) || off4(beta) || off4(mean) || off4(rstd) ||
        reinterpret_cast<uintptr_t>(workspace) % 16)
        return PP_ERR_ALIGN;
    const Space w = space_of(s, false);
    if (workspace_bytes < w.bytes()) return PP_ERR_BUFFER;
    const size_t yb = (size_t)N * pixels * C * size_of(dtype);
    // y may be x itself where x is dense: every value is read before it is written
    if (!(x == y && x_pixel == C && x_sample == pixels * C) && overlap(x, extent(s, x_pixel, x_sample), y, yb))
        return PP_ERR_BUFFER;
    const Split p = split_of(s, std::min({align_of(x), align_of(y), align_of(C, dtype),
                                          pixels > 1 ? align_of(x_pixel, dtype) : 16,
                                          N > 1 ? align_of(x_sample, dtype) : 16}));
    NormArgs a{};
    take(a, s, p);
    a.x = x;
    a.x_pixel = x_pixel;
    a.x_sample = x_sample;
    a.gamma = gamma;
    a.beta = beta;
    a.eps = eps;
    a.act = act;
    a.out = y;
    a.parts = static_cast<float*>(workspace);
    a.mean_out = mean ? mean : a.parts + w.parts;
    a.rstd_out = rstd ? rstd : a.parts + w.parts + (size_t)N * G;
    a.mean = a.mean_out;
    a.rstd = a.rstd_out;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == PP_F32   ? forward<float>(a, p.V, st)
                          : dtype == PP_F16 ? forward<__half>(a, p.V, st)
                                            : forward<__nv_bfloat16>(a, p.V, st);
    return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

int pp_group_norm_backward(const void* dy, int64_t dy_pixel, int64_t dy_sample, const void* x, int64_t x_pixel,
                           int64_t x_sample, int dtype, int N, int64_t pixels, int C, int G, const float* gamma,
                           const float* beta, const float* mean, const float* rstd, int act, void* dx, float* dgamma,
                           float* dbeta, void* workspace, size_t workspace_bytes, void* stream) {
    const Shape s{dtype, N, C, G, pixels};
    if (const int e = check_shape(s)) return e;
    if (act != PP_ACT_NONE && act != PP_ACT_RELU && act != PP_ACT_SILU) return PP_ERR_ARG;
    if (off4(gamma) || off4(beta) || off4(mean) || off4(rstd) || off4(dgamma) || off4(dbeta)) return PP_ERR_ALIGN;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!N || !pixels) {                            // sums over nothing
        if (dgamma && cudaMemsetAsync(dgamma, 0, (size_t)C * 4, st) != cudaSuccess) return PP_ERR_CUDA;
        if (dbeta && cudaMemsetAsync(dbeta, 0, (size_t)C * 4, st) != cudaSuccess) return PP_ERR_CUDA;
        return PP_OK;
    }
    if (const int e = check_input(s, dy, dy_pixel, dy_sample)) return e;
    if (const int e = check_input(s, x, x_pixel, x_sample)) return e;
    if (!mean || !rstd || !dx || !workspace) return PP_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(dx) % size_of(dtype) || reinterpret_cast<uintptr_t>(workspace) % 16)
        return PP_ERR_ALIGN;
    const Space w = space_of(s, true);
    if (workspace_bytes < w.bytes()) return PP_ERR_BUFFER;
    const size_t xb = (size_t)N * pixels * C * size_of(dtype);
    const bool over_dy = dx == dy && dy_pixel == C && dy_sample == pixels * C;
    if (overlap(x, extent(s, x_pixel, x_sample), dx, xb) ||
        (!over_dy && overlap(dy, extent(s, dy_pixel, dy_sample), dx, xb)))
        return PP_ERR_BUFFER;
    const Split p = split_of(s, std::min({align_of(x), align_of(dy), align_of(dx), align_of(C, dtype),
                                          pixels > 1 ? align_of(x_pixel, dtype) : 16,
                                          pixels > 1 ? align_of(dy_pixel, dtype) : 16,
                                          N > 1 ? align_of(x_sample, dtype) : 16,
                                          N > 1 ? align_of(dy_sample, dtype) : 16}));
    NormArgs a{};
    take(a, s, p);
    a.x = x;
    a.x_pixel = x_pixel;
    a.x_sample = x_sample;
    a.dy = dy;
    a.dy_pixel = dy_pixel;
    a.dy_sample = dy_sample;
    a.gamma = gamma;
    a.beta = beta;
    a.act = act;
    a.mean = mean;
    a.rstd = rstd;
    a.out = dx;
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.parts = static_cast<float*>(workspace);
    a.sums = a.parts + w.parts;
    const cudaError_t e = dtype == PP_F32   ? backward<float>(a, p.V, st)
                          : dtype == PP_F16 ? backward<__half>(a, p.V, st)
                                            : backward<__nv_bfloat16>(a, p.V, st);
    return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

}  // extern "C"
