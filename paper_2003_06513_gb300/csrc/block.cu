// Block norm: what joins a block's output to the residual stream and hands the stream to the next block, on
// channels-last activations, for retraining residual nets.  Plans, the join of the gradients' sums, C entry points
// (kernels: block.cuh).
//
// For every pixel, over its C channels, with a norm v^ = (v - mean) / sqrt(mean (v - mean)^2 + eps), mean 0 in a norm by the
// root of the mean square,
//     u = post_weight b^ + post_bias,   h = x + scale gate_n u,   z = weight h^ + bias,   y = act(z);
// backward, with dz = dy act'(z), t = dz weight and M over the channels,
//     dx = dh + (t - M t - h^ M(t h^)) / root_h,
//     db = (s - M s - b^ M(s b^)) / root_b,   s = dx scale gate_n post_weight,
// (M t and M s only where the norm takes the mean out), and of the parameters, from the sums over a sample's pixels
// e = sum dx b^ and f = sum dx:   joined_n = post_weight e + post_bias f,
//     dgate_n = scale joined_n,  dscale = sum_n gate_n joined_n,  dpost_weight = sum_n scale gate_n e,  dpost_bias with f,
//     dweight = sum dz h^,  dbias = sum dz.
//
// Memory would bound it: four arrays forward, six backward.  What does is latency: a row's chain of readings, shuffles and 20 to 60
// operations a value, each of which waits for the one before, at the 24 (forward) and 16 (backward) warps of an SM that the
// registers allow; 52 to 55 % of the issue slots are used, and no single wait stands out.  Forward 32 x 256 x 56 x 56 fp16, layer
// norms, ReLU and a gate, takes 41 us, 5.1 TB/s, 0.75 of a copy's rate; backward 32 x 128 x 112 x 112 124 us, 5.0 TB/s, 0.73; RMS
// norms 41 and 109, of fp32 backward 204 (0.89).  (GPU time, calls one after another in one graph.)  Mean and root are not kept for the backward pass, which
// has h and b in registers anyway.  A CTA takes a stretch of consecutive pixels (the gate is read when the sample changes,
// not with each row) and in the backward pass keeps its channels' sums in registers; the CTAs' sums are joined by a second
// launch, in order, which is started before the first one's end (norm_starts_early).  By loads that are waited for, with any
// strides and kinds in each loop, the two took 90 and 228 us.
#include <algorithm>
#include <climits>
#include <cmath>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "block.h"
#include "norm.h"
#include "patconv.h"

namespace patconv {

extern template struct BlockKernels<float, float>;
extern template struct BlockKernels<__half, __half>;
extern template struct BlockKernels<__nv_bfloat16, __nv_bfloat16>;
extern template struct BlockKernels<float, __half>;
extern template struct BlockKernels<float, __nv_bfloat16>;

namespace {

constexpr int kSMs = 152;

int row_threads(int C) {
    const int need = (C + kBlockEight - 1) / kBlockEight;
    if (need > 32) return (need + 31) / 32 * 32;
    int t = 1;
    while (t < need) t *= 2;
    return t;
}

constexpr int kJoinChannels = 32, kJoinParts = 32;

// The gate's gradient of sample y has parts of several CTAs: adds those from part `k0` on, every step-th, of channel c.  With more
// samples than CTAs y is a CTA, and the sample the one that begins in it and ends in another.  Whether there is one.
struct GateParts {
    const float* own;                                 // the first part: the CTA's only, or the second of its two places
    const float* from;                                // and the others
    float* to;
    int n;
    __device__ __forceinline__ bool find(const BlockArgs& a, int64_t y) {
        const int64_t i = a.N <= a.ctas ? y * a.pixels / a.stretch : y;
        const int64_t begin = i * a.stretch, end = begin + a.stretch;
        if (end >= a.rows) return false;              // the last CTA's samples end there
        const int64_t sample = a.N <= a.ctas ? y : (end - 1) / a.pixels, first = sample * a.pixels, last = first + a.pixels;
        if (last <= end || first < begin) return false;       // it ends with this CTA, or began in an earlier one
        own = a.gates + (i * 2 + (first > begin)) * a.C;
        from = a.gates + (i + 1) * 2 * a.C;           // of those the sample is the first
        to = a.dgate + sample * a.C;
        n = (int)((last - 1) / a.stretch - i);
        return true;
    }
};
// samples of a CTA of the join: one, whose parts its threads share, or, where a sample has few parts, one for each of its rows of
// threads (32 x 2048 x 7 x 7, eight parts: 23 us by CTAs of their own; but 32 x 24 x 112 x 112, 19 parts, takes 4 us more so)
constexpr int kFewParts = 10;
__host__ __device__ inline int samples_of_join(const BlockArgs& a) { return a.pixels <= (int64_t)kFewParts * a.stretch ? kJoinParts : 1; }

// Sums of the CTAs' parts: blockIdx.y below kBlockSums one of the sums over all rows, else the gate's gradients of samples that
// several CTAs have parts of.
__global__ void __launch_bounds__(kJoinChannels* kJoinParts) block_sums(BlockArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");        // its launch overlaps the end of the kernel before it
    __shared__ float parts[kJoinParts][kJoinChannels + 1];
    const int c = blockIdx.x * kJoinChannels + threadIdx.x % kJoinChannels, part = threadIdx.x / kJoinChannels;
    const int64_t step = (blockIdx.y < kBlockSums ? kBlockSums : 2) * (int64_t)a.C;
    GateParts gate;
    float s = 0;
    if (blockIdx.y < kBlockSums) {
        float* const all[kBlockSums] = {a.dweight, a.dbias, a.dpost_weight, a.dpost_bias, a.dscale};
        gate.to = all[blockIdx.y];
        if (!gate.to) return;
        gate.from = a.sums + (int64_t)blockIdx.y * a.C;
        gate.n = a.ctas;
    } else if (samples_of_join(a) > 1) {
        const int64_t y = (int64_t)(blockIdx.y - kBlockSums) * kJoinParts + part;
        if (y >= min(a.N, a.ctas) || c >= a.C || !gate.find(a, y)) return;
        s = gate.own[c];
#pragma unroll 8
        for (int k = 0; k < gate.n; ++k) s += gate.from[k * step + c];
        gate.to[c] = s;
        return;
    } else {
        if (!gate.find(a, blockIdx.y - kBlockSums)) return;
        if (c < a.C && part == 0) s = gate.own[c];
    }
    if (c < a.C)
#pragma unroll 8
        for (int k = part; k < gate.n; k += kJoinParts) s += gate.from[k * step + c];
    parts[part][threadIdx.x % kJoinChannels] = s;
    __syncthreads();
    if (part || c >= a.C) return;
    s = 0;
    for (int p = 0; p < kJoinParts; ++p) s += parts[p][threadIdx.x];
    gate.to[c] = s;
}

int size_of(int dtype) { return dtype == PP_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == PP_F32 || dtype == PP_F16 || dtype == PP_BF16; }
bool off(const void* p, size_t align) { return reinterpret_cast<uintptr_t>(p) % align != 0; }
bool overlap(const void* a, size_t an, const void* b, size_t bn) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && an && bn && x < y + bn && y < x + an;
}

struct Shape {
    int x_dtype, dtype, N, C;
    int64_t pixels;
};
struct Input {
    const void* p;
    int64_t pixel, sample;
    int es;
    bool dense(const Shape& s) const {
        return (s.pixels == 1 || pixel == s.C) && (s.N == 1 || sample == s.pixels * s.C);
    }
    size_t bytes(const Shape& s) const { return (size_t)((s.N - 1) * sample + (s.pixels - 1) * pixel + s.C) * es; }
    // the largest of 8, 4, 2 and 1 channels that a vector of it can have
    int vector(const Shape& s) const {
        for (const int v : {8, 4, 2}) {
            const size_t align = std::min(16, v * es);
            if (s.C % v == 0 && !off(p, align) && (s.pixels == 1 || pixel * es % align == 0) && (s.N == 1 || sample * es % align == 0)) return v;
        }
        return 1;
    }
};

int check_shape(const Shape& s) {
    if (!known(s.x_dtype) || !known(s.dtype) || (s.x_dtype != s.dtype && s.x_dtype != PP_F32)) return PP_ERR_DTYPE;
    if (s.N < 0 || s.pixels < 0 || s.C < 1 || s.C > kBlockMost) return PP_ERR_SHAPE;
    if (s.N && s.pixels && s.pixels > (INT_MAX - (1 << 24)) / s.N) return PP_ERR_SHAPE;     // (a CTA's last row and its rounds fit too)
    return PP_OK;
}
int check_input(const Shape& s, const Input& t) {
    if (!t.p) return PP_ERR_NULL;
    if (off(t.p, t.es)) return PP_ERR_ALIGN;
    if ((s.pixels > 1 && t.pixel < s.C) || (s.N > 1 && t.sample < 0) || t.pixel > INT_MAX || t.sample > (int64_t(1) << 50) / s.N)
        return PP_ERR_SHAPE;
    return PP_OK;
}
int check_kinds(int post, int pre, int act, float eps) {
    for (const int k : {post, pre})
        if (k != PP_NORM_NONE && k != PP_NORM_RMS && k != PP_NORM_LAYER) return PP_ERR_ARG;
    if (act != PP_ACT_NONE && act != PP_ACT_RELU && act != PP_ACT_SILU) return PP_ERR_ARG;
    if (pre == PP_NORM_NONE && act != PP_ACT_NONE) return PP_ERR_ARG;
    return eps >= 0 && std::isfinite(eps) ? PP_OK : PP_ERR_ARG;
}
bool odd(std::initializer_list<const float*> all) {
    for (const float* p : all)
        if (off(p, 4)) return true;
    return false;
}

BlockArgs args_of(const Shape& s, const float* post_weight, const float* post_bias, const float* scale, const float* gate, int post,
                  int pre, const float* weight, const float* bias, int act, float eps) {
    BlockArgs a{};
    a.post_weight = post_weight;
    a.post_bias = post_bias;
    a.scale = scale;
    a.gate = gate;
    a.weight = weight;
    a.bias = bias;
    a.post = post;
    a.pre = pre;
    a.act = act;
    a.eps = eps;
    a.inv_c = 1.0f / (float)s.C;
    a.rows = (int)(s.N * s.pixels);
    a.C = s.C;
    a.N = s.N;
    a.pixels = s.pixels;
    int bits = 0;
    while ((int64_t(1) << bits) < s.pixels) ++bits;
    a.pixels_shift = 31 + bits;
    a.pixels_mul = s.pixels > 1 ? (uint32_t)(((uint64_t(1) << a.pixels_shift) + s.pixels - 1) / s.pixels) : 0;
    a.threads = row_threads(s.C);
    a.ragged = a.threads * kBlockEight != s.C;
    a.flat = a.dense = 1;
    return a;
}
void set(BlockArgs& a, const void* BlockArgs::*p, int64_t BlockArgs::*pixel, int64_t BlockArgs::*sample, const Input& t) {
    if (t.p && a.N > 1 && t.sample != a.pixels * t.pixel) a.flat = 0;
    if (t.p && !t.dense(Shape{0, 0, a.N, a.C, a.pixels})) a.dense = 0;
    a.*p = t.p;
    a.*pixel = t.pixel;
    a.*sample = t.sample;
}
// of results, whose rows are dense
int vector_of(const Shape& s, const void* p, int es) { return p ? Input{p, s.C, s.pixels * s.C, es}.vector(s) : 8; }

// what there are kernels for: eight where both are of two bytes, else four; two; one
int known_vector(const Shape& s, int v) {
    if (s.x_dtype == PP_F32) return v >= 4 ? 4 : v;
    return v == 8 ? 8 : std::min(v, 2);
}

template <typename F>
int by_type(const Shape& s, F&& f) {
    const cudaError_t e = s.dtype == PP_F32   ? f(BlockKernels<float, float>())
                          : s.dtype == PP_F16 ? (s.x_dtype == PP_F16 ? f(BlockKernels<__half, __half>()) : f(BlockKernels<float, __half>()))
                          : s.x_dtype == PP_BF16 ? f(BlockKernels<__nv_bfloat16, __nv_bfloat16>())
                                                 : f(BlockKernels<float, __nv_bfloat16>());
    return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

size_t workspace_of(const Shape& s) {
    int64_t stretch;
    return s.N && s.pixels ? (size_t)block_ctas(s.N * s.pixels, s.C, &stretch) * (kBlockSums + 2) * s.C * sizeof(float) : 0;
}

}  // namespace

// One wave of CTAs: four of 128 threads on an SM, of 128 registers a thread, or as many of longer rows' threads.  (Backward 32 x
// 128 x 112 x 112 fp16 127 us; with 80 registers a thread, for six CTAs, 217, as they spill.)
int block_ctas(int64_t rows, int C, int64_t* stretch) {
    const int threads = row_threads(C), here = threads > 32 ? 1 : kBlockBackThreads / threads;
    const int64_t most = threads > 32 ? kSMs * std::max(1, 512 / threads) : kSMs * 4;
    const int64_t n = std::min(most, (rows + here - 1) / here);
    *stretch = (rows + n - 1) / n;
    return (int)((rows + *stretch - 1) / *stretch);
}

cudaError_t block_join(const BlockArgs& a, cudaStream_t st) {
    if (!a.dweight && !a.dbias && !a.dpost_weight && !a.dpost_bias && !a.dscale && !a.dgate) return cudaSuccess;
    const dim3 grid((a.C + kJoinChannels - 1) / kJoinChannels, kBlockSums + (a.dgate ? (std::min(a.N, a.ctas) + samples_of_join(a) - 1) / samples_of_join(a) : 0));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kJoinChannels * kJoinParts);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = norm_starts_early();
    const cudaError_t e = cudaLaunchKernelEx(&cfg, block_sums, a), l = cudaGetLastError();
    return e != cudaSuccess ? e : l;
}

}  // namespace patconv

using namespace patconv;

extern "C" {

int pp_block_norm_workspace_size(int N, int64_t pixels, int C, size_t* bytes) {
    if (!bytes) return PP_ERR_NULL;
    const Shape s{PP_F32, PP_F32, N, C, pixels};
    if (const int e = check_shape(s)) return e;
    *bytes = workspace_of(s);
    return PP_OK;
}

int pp_block_norm(const void* x, int64_t x_pixel, int64_t x_sample, int x_dtype, const void* block, int64_t block_pixel,
                  int64_t block_sample, int dtype, int N, int64_t pixels, int C, int post, const float* post_weight,
                  const float* post_bias, const float* scale, const float* gate, int pre, const float* weight, const float* bias,
                  int act, float eps, void* h, void* y, void* stream) {
    const Shape s{x_dtype, dtype, N, C, pixels};
    if (const int e = check_shape(s)) return e;
    if (const int e = check_kinds(post, pre, act, eps)) return e;
    if (odd({post_weight, post_bias, scale, gate, weight, bias})) return PP_ERR_ALIGN;
    if ((post == PP_NORM_NONE && (post_weight || post_bias)) || (pre == PP_NORM_NONE && (weight || bias))) return PP_ERR_ARG;
    if (!N || !pixels) return PP_OK;                  // (of no values there are no addresses to go by)
    if (!block && (post != PP_NORM_NONE || scale || gate || pre == PP_NORM_NONE)) return PP_ERR_ARG;
    const Input in{x, x_pixel, x_sample, size_of(x_dtype)}, b{block, block_pixel, block_sample, size_of(dtype)};
    if (const int e = check_input(s, in)) return e;
    if (block)
        if (const int e = check_input(s, b)) return e;
    if ((block && !h) || (pre != PP_NORM_NONE && !y)) return PP_ERR_NULL;
    if (!block) h = nullptr;
    if (pre == PP_NORM_NONE) y = nullptr;
    if (off(h, in.es) || off(y, b.es)) return PP_ERR_ALIGN;
    const size_t values = (size_t)N * pixels * C, hb = h ? values * in.es : 0, yb = y ? values * b.es : 0;
    // h may be x itself, and y the block's output, where those are dense: every value is read before it is written
    if ((!(h == x && in.dense(s)) && overlap(h, hb, x, in.bytes(s))) || (block && overlap(h, hb, block, b.bytes(s))) ||
        (block && !(y == block && b.dense(s)) && overlap(y, yb, block, b.bytes(s))) || overlap(y, yb, x, in.bytes(s)) || overlap(h, hb, y, yb))
        return PP_ERR_BUFFER;
    BlockArgs a = args_of(s, post_weight, post_bias, scale, gate, post, pre, weight, bias, act, eps);
    set(a, &BlockArgs::x, &BlockArgs::x_pixel, &BlockArgs::x_sample, in);
    set(a, &BlockArgs::b, &BlockArgs::b_pixel, &BlockArgs::b_sample, b);
    a.h = h;
    a.y = y;
    a.full = block != nullptr;
    const int V = known_vector(s, std::min({in.vector(s), block ? b.vector(s) : 8, vector_of(s, h, in.es), vector_of(s, y, b.es)}));
    a.vectors = C / V;
    return by_type(s, [&](auto k) { return k.forward(a, V, static_cast<cudaStream_t>(stream)); });
}

int pp_block_norm_backward(const void* dh, int64_t dh_pixel, int64_t dh_sample, const void* dy, int64_t dy_pixel, int64_t dy_sample,
                           const void* h, int64_t h_pixel, int64_t h_sample, int x_dtype, const void* block, int64_t block_pixel,
                           int64_t block_sample, int dtype, int N, int64_t pixels, int C, int post, const float* post_weight,
                           const float* post_bias, const float* scale, const float* gate, int pre, const float* weight,
                           const float* bias, int act, float eps, void* dx, void* dblock, float* dpost_weight, float* dpost_bias,
                           float* dscale, float* dgate, float* dweight, float* dbias, void* workspace, size_t workspace_bytes,
                           void* stream) {
    const Shape s{x_dtype, dtype, N, C, pixels};
    if (const int e = check_shape(s)) return e;
    if (const int e = check_kinds(post, pre, act, eps)) return e;
    if (odd({post_weight, post_bias, scale, gate, weight, bias, dpost_weight, dpost_bias, dscale, dgate, dweight, dbias})) return PP_ERR_ALIGN;
    if ((post == PP_NORM_NONE && (post_weight || post_bias || dpost_weight || dpost_bias)) ||
        (pre == PP_NORM_NONE && (weight || bias || dweight || dbias)))
        return PP_ERR_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!N || !pixels) {                              // sums over nothing
        for (float* p : {dpost_weight, dpost_bias, dscale, dweight, dbias, dgate})
            if (p && (p != dgate || N) && cudaMemsetAsync(p, 0, (size_t)C * (p == dgate ? N : 1) * 4, st) != cudaSuccess) {
                cudaGetLastError();
                return PP_ERR_CUDA;
            }
        return PP_OK;
    }
    if (!block && (post != PP_NORM_NONE || scale || gate || dpost_weight || dpost_bias || dscale || dgate)) return PP_ERR_ARG;
    if ((pre == PP_NORM_NONE && dy) || (!gate && dgate)) return PP_ERR_ARG;
    const int xs = size_of(x_dtype), bs = size_of(dtype);
    const Input d{dh, dh_pixel, dh_sample, xs}, e{dy, dy_pixel, dy_sample, bs}, in{h, h_pixel, h_sample, xs}, b{block, block_pixel, block_sample, bs};
    const bool norm = pre != PP_NORM_NONE && dy;      // without a gradient of y its norm has none either
    for (const Input* t : {&d, &e, &in, &b})
        if (t->p && (t != &in || norm))
            if (const int err = check_input(s, *t)) return err;
    if (!dx || (block && !dblock) || !workspace || (norm && !h)) return PP_ERR_NULL;
    if (off(dx, xs) || off(dblock, bs) || off(workspace, 16)) return PP_ERR_ALIGN;
    if (workspace_bytes < workspace_of(s)) return PP_ERR_BUFFER;
    if (!block) dblock = nullptr;
    const size_t values = (size_t)N * pixels * C, xb = values * xs, bb = dblock ? values * bs : 0;
    // dx may be dh itself, and dblock dy, where those are dense: every value is read before it is written
    if (overlap(dx, xb, dblock, bb)) return PP_ERR_BUFFER;
    for (const Input* t : {&d, &e, &in, &b}) {
        if (!t->p || (t == &in && !norm)) continue;
        const size_t n = t->bytes(s);
        if ((overlap(dx, xb, t->p, n) && !(t == &d && dx == dh && d.dense(s))) ||
            (overlap(dblock, bb, t->p, n) && !(t == &e && dblock == dy && e.dense(s))))
            return PP_ERR_BUFFER;
    }
    BlockArgs a = args_of(s, post_weight, post_bias, scale, gate, post, norm ? pre : PP_NORM_NONE, weight, bias, norm ? act : PP_ACT_NONE, eps);
    set(a, &BlockArgs::dh, &BlockArgs::dh_pixel, &BlockArgs::dh_sample, d);
    set(a, &BlockArgs::dy, &BlockArgs::dy_pixel, &BlockArgs::dy_sample, e);
    set(a, &BlockArgs::x, &BlockArgs::x_pixel, &BlockArgs::x_sample, in);
    set(a, &BlockArgs::b, &BlockArgs::b_pixel, &BlockArgs::b_sample, b);
    a.dx = dx;
    a.db = dblock;
    a.dweight = dweight;
    a.dbias = dbias;
    a.dpost_weight = dpost_weight;
    a.dpost_bias = dpost_bias;
    a.dscale = dscale;
    a.dgate = dgate;
    int V = std::min(vector_of(s, dx, xs), vector_of(s, dblock, bs));
    for (const Input* t : {&d, &e, &in, &b})
        if (t->p && (t != &in || norm)) V = std::min(V, t->vector(s));
    V = known_vector(s, V);
    a.vectors = C / V;
    a.full = block && dh && norm;
    int64_t stretch;
    a.ctas = block_ctas((int64_t)N * pixels, C, &stretch);
    a.stretch = (int)stretch;
    a.sums = static_cast<float*>(workspace);
    a.gates = a.sums + (size_t)a.ctas * kBlockSums * C;
    return by_type(s, [&](auto k) { return k.backward(a, V, st); });
}

}  // extern "C"
