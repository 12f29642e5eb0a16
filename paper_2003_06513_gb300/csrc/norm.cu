// Group norm with its activation on channels-last activations, forward and backward, for masked
// retraining: plans and C entry points (kernels: norm.cuh).
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
// Resident form: a cluster of up to 8 CTAs takes a unit -- whole groups of one sample, a slab of channels
// of 32 to 128 bytes -- and holds it in registers between the sums and the result, the CTAs' sums being
// joined through distributed shared memory, so that every value is read from memory once.
// Streamed form, for units that 8 CTAs do not hold: one persistent kernel whose CTAs take stretches of
// pixels, for a sample's sums first and some samples later for its result, so that the second reading
// comes from L2.
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
#include <numeric>

#include "norm.h"
#include "patconv.h"

namespace patconv {

extern template struct NormKernels<float>;
extern template struct NormKernels<__half>;
extern template struct NormKernels<__nv_bfloat16>;

namespace {

struct Shape {
    int dtype, N, C, G;
    int64_t pixels;
    bool backward;
};

int size_of(int dtype) { return dtype == PP_F32 ? 4 : 2; }

int check_shape(const Shape& s) {
    if (s.dtype != PP_F32 && s.dtype != PP_F16 && s.dtype != PP_BF16) return PP_ERR_DTYPE;
    if (s.N < 0 || s.N > 65534 || s.C < 1 || s.C > (1 << 20) || s.G < 1 || s.C % s.G || s.pixels < 0 ||
        s.pixels > INT_MAX)
        return PP_ERR_SHAPE;
    if (s.N && s.pixels && s.pixels > (int64_t(1) << 42) / s.N / s.C) return PP_ERR_SHAPE;
    return PP_OK;
}

struct Plan {
    int V = 1;                              // channels of a thread's vector
    int cols = 1, rows = 1, chunk = 1;      // vectors of a row and rows of a CTA, pixels of a CTA
    int NS = 1;                             // sets of a vector's channels that are summed apart
    int tiles = 1, chunks = 1, ahead = 1, draw = 1, grid = 1;   // streamed: CTAs side by side, stretches down a sample
    int K = 0, cluster = 1, slabs = 1;   // resident: vectors held (0: streamed), CTAs a unit, slabs
    size_t parts = 0, sums = 0;             // floats of the workspace
};

constexpr int kSMs = 152;
constexpr int kStretch = 131072;

// The resident form: the narrowest slab of whole groups that is 128 bytes wide or a whole row, or if that
// is too much for 8 CTAs, narrower ones down to a 32-byte sector; no more CTAs than hold it at 8 vectors of
// 16 bytes a thread (3 CTAs an SM; 16 vectors let in 2), but enough for the GPU's SMs.
bool resident(const Shape& s, Plan& p) {
    const int es = size_of(s.dtype), bytes = p.V * es, cpg = s.C / s.G, vectors = s.C / p.V;
    const int unit = std::lcm(cpg, p.V) / p.V;              // vectors of the least slab of whole groups
    if (unit > kNormThreads || vectors % unit) return false;
    const bool wide = bytes == 16;
    const int *held = wide ? (s.backward ? kHeldBackWide : kHeldWide) : (s.backward ? kHeldBackSmall : kHeldSmall);
    const int n_held = wide ? (s.backward ? 3 : 4) : 2, most = held[n_held - 1];
    const int steps = vectors / unit;
    int best = 0, best_cluster = 0;
    const auto needs = [&](int cols, int cluster) {         // vectors a thread
        const int rows = kNormThreads / cols;
        const int64_t chunk = (s.pixels + cluster - 1) / cluster;
        return (chunk + rows - 1) / rows;
    };
    const auto cluster_of = [&](int cols, int limit) {      // CTAs that hold it with `limit` vectors a thread
        for (int c = 1; c <= 8; c *= 2)
            if (needs(cols, c) <= limit) return c;
        return 0;
    };
    for (int m = 1; m <= steps; ++m) {                      // widths upwards
        if (steps % m || m * unit > kNormThreads || m * unit * p.V > 1024) continue;
        const int width = m * unit * bytes, c = cluster_of(m * unit, most);
        if (width < 32 && m < steps) continue;
        if (!c) break;                                      // wider ones need more still
        best = m * unit;
        best_cluster = c;
        if (width >= 128) break;
    }
    if (!best) return false;
    if (const int c = cluster_of(best, std::min(most, wide ? 8 : most))) best_cluster = c;
    p.cols = best;
    p.rows = kNormThreads / best;
    p.slabs = vectors / best;
    while (best_cluster < 8 && (int64_t)s.N * p.slabs * best_cluster < kSMs && needs(best, best_cluster) > 2) best_cluster *= 2;
    if (p.slabs > 65535) return false;                      // the grid's second dimension
    p.cluster = best_cluster;
    p.chunk = (int)((s.pixels + best_cluster - 1) / best_cluster);
    p.K = *std::find_if(held, held + n_held, [&](int k) { return k >= needs(best, best_cluster); });
    p.parts = s.backward ? (size_t)s.N * best_cluster * s.C * 2 : 0;
    return true;
}

// V channels a thread (16 bytes where `align`, the common alignment of addresses and strides in bytes,
// allows it, else 4 bytes or one channel).  Streamed: a row's vectors over the threads of one or more CTAs,
// stretches of pixels of about kStretch bytes of each input, and as many samples ahead as the CTAs at work
// need, so that none waits for a sample's sums.
Plan plan_of(const Shape& s, int align) {
    Plan p;
    const int es = size_of(s.dtype), cpg = s.C / s.G;
    p.V = align >= 16 ? 16 / es : std::max(1, std::min(align, 4) / es);
    p.NS = cpg % p.V ? p.V : 1;
    if (!resident(s, p)) {
        const int vectors = s.C / p.V;
        p.tiles = (vectors + kNormThreads - 1) / kNormThreads;
        p.cols = (vectors + p.tiles - 1) / p.tiles;
        p.rows = kNormThreads / p.cols;
        const int64_t row = (int64_t)p.cols * p.V * es;
        const int64_t wanted = std::max<int64_t>((kStretch + row - 1) / row, p.rows);
        p.chunks = (int)((s.pixels + wanted - 1) / wanted);
        p.chunk = (int)((s.pixels + p.chunks - 1) / p.chunks);
        p.chunks = (int)((s.pixels + p.chunk - 1) / p.chunk);
        // batches of the last, smallest stretch: the load side is at most kStreamDepth - 1 batches ahead
        const int batch = p.rows * (s.backward ? kStreamBatch / 2 : kStreamBatch);
        const int least = (int)((s.pixels - (int64_t)(p.chunks - 1) * p.chunk + batch - 1) / batch);
        p.draw = (kStreamDepth - 2 + least) / least + 1;
        const int64_t per = (int64_t)p.chunks * p.tiles;
        p.grid = (int)std::min<int64_t>(2 * per * s.N, kSMs * 2);
        p.ahead = (int)std::min<int64_t>(s.N, 1 + (2 * (int64_t)p.grid + per - 1) / per);
        const size_t sets = s.backward ? s.C : s.C / (p.V / p.NS);
        p.parts = (size_t)s.N * p.chunks * sets * 2;
        p.sums = (s.backward ? (size_t)s.N * s.C * 2 + (size_t)s.N * s.G * 2 : 0) + (norm_counters(s.N) + 1) / 2 * 2;
    }
    if (!s.backward) p.sums += (size_t)s.N * s.G * 2;       // mean and rstd that the caller does not want
    return p;
}

// of any plan that a call's alignment may lead to
size_t workspace_of(const Shape& s) {
    size_t most = 0;
    for (int align = size_of(s.dtype); align <= 16; align *= 2)
        if ((int64_t)s.C * size_of(s.dtype) % align == 0) {
            const Plan p = plan_of(s, align);
            most = std::max(most, (p.parts + p.sums) * sizeof(float));
        }
    return most;
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
cudaError_t run(const NormArgs& a, const Plan& p, bool backward, cudaStream_t st) {
    using K = NormKernels<T>;
    return backward ? K::backward(a, p.V, p.K, st) : K::forward(a, p.V, p.NS, p.K, st);
}

NormArgs args_of(const Shape& s, const Plan& p, const void* x, int64_t x_pixel, int64_t x_sample, const float* gamma,
                 const float* beta, int act, void* out, void* workspace) {
    NormArgs a{};
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
    a.ahead = p.ahead;
    a.draw = p.draw;
    a.grid = p.grid;
    a.cluster = p.cluster;
    a.slabs = p.slabs;
    a.groups = p.cols * p.V / a.cpg;
    a.spg = a.cpg / (p.V / p.NS);
    const auto inverse = [](int d) { return d > 1 ? (uint32_t)(((uint64_t(1) << 32) + d - 1) / d) : 0; };
    a.spg_mul = inverse(a.spg);
    a.cpg_mul = inverse(a.cpg);
    a.cols_mul = inverse(a.cols);
    a.rows_mul = inverse(a.rows);
    a.x = x;
    a.x_pixel = x_pixel;
    a.x_sample = x_sample;
    a.gamma = gamma;
    a.beta = beta;
    a.act = act;
    a.out = out;
    a.parts = static_cast<float*>(workspace);
    a.counters = reinterpret_cast<uint32_t*>(a.parts + p.parts);
    return a;
}

int done(NormArgs& a, const Plan& p, const Shape& s, void* stream) {
    if (!p.K && !(a.status = device_status_word())) return PP_ERR_CUDA;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = s.dtype == PP_F32   ? run<float>(a, p, s.backward, st)
                          : s.dtype == PP_F16 ? run<__half>(a, p, s.backward, st)
                                              : run<__nv_bfloat16>(a, p, s.backward, st);
    return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

bool off4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; }

}  // namespace
}  // namespace patconv

using namespace patconv;

extern "C" {

int pp_group_norm_workspace_size(int dtype, int N, int64_t pixels, int C, int G, int backward, size_t* bytes) {
    if (!bytes) return PP_ERR_NULL;
    const Shape s{dtype, N, C, G, pixels, backward == 1};
    if (const int e = check_shape(s)) return e;
    if (backward != 0 && backward != 1) return PP_ERR_ARG;
    *bytes = N && pixels ? workspace_of(s) : 0;
    return PP_OK;
}

int pp_group_norm_plan(int dtype, int N, int64_t pixels, int C, int G, int backward, int align, int64_t* info, int n_info) {
    if (!info) return PP_ERR_NULL;
    const Shape s{dtype, N, C, G, pixels, backward == 1};
    if (const int e = check_shape(s)) return e;
    if ((backward != 0 && backward != 1) || align < size_of(dtype) || (align & (align - 1)) || n_info < 0) return PP_ERR_ARG;
    if (!N || !pixels) return PP_ERR_SHAPE;
    int common = align < 16 ? align : 16;
    while ((int64_t)C * size_of(dtype) % common) common /= 2;
    const Plan p = plan_of(s, common);
    const int64_t all[8] = {p.K ? 2 : 1, p.V, p.cols, p.chunk, p.K, p.cluster,
                            p.K ? (int64_t)N * p.slabs * p.cluster : p.grid, p.NS};
    for (int i = 0; i < n_info && i < 8; ++i) info[i] = all[i];
    return PP_OK;
}

int pp_group_norm(const void* x, int64_t x_pixel, int64_t x_sample, int dtype, int N, int64_t pixels, int C, int G,
                  const float* gamma, const float* beta, float eps, int act, void* y, float* mean, float* rstd,
                  void* workspace, size_t workspace_bytes, void* stream) {
    const Shape s{dtype, N, C, G, pixels, false};
    if (const int e = check_shape(s)) return e;
    if (act != PP_ACT_NONE && act != PP_ACT_RELU && act != PP_ACT_SILU) return PP_ERR_ARG;
    if (!(eps >= 0) || !std::isfinite(eps)) return PP_ERR_ARG;
    if (!N || !pixels) return PP_OK;
    if (const int e = check_input(s, x, x_pixel, x_sample)) return e;
    if (!y || !workspace) return PP_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(y) % size_of(dtype) || off4(gamma) || off4(beta) || off4(mean) || off4(rstd) ||
        reinterpret_cast<uintptr_t>(workspace) % 16)
        return PP_ERR_ALIGN;
    if (workspace_bytes < workspace_of(s)) return PP_ERR_BUFFER;
    const size_t yb = (size_t)N * pixels * C * size_of(dtype);
    // y may be x itself where x is dense: every value is read before it is written
    if (!(x == y && x_pixel == C && x_sample == pixels * C) && overlap(x, extent(s, x_pixel, x_sample), y, yb))
        return PP_ERR_BUFFER;
    const Plan p = plan_of(s, std::min({align_of(x), align_of(y), align_of(C, dtype),
                                          pixels > 1 ? align_of(x_pixel, dtype) : 16,
                                          N > 1 ? align_of(x_sample, dtype) : 16}));
    NormArgs a = args_of(s, p, x, x_pixel, x_sample, gamma, beta, act, y, workspace);
    a.eps = eps;
    float* own = a.parts + p.parts + p.sums - 2 * (size_t)N * G;
    a.mean_out = mean ? mean : own;
    a.rstd_out = rstd ? rstd : own + (size_t)N * G;
    return done(a, p, s, stream);
}

int pp_group_norm_backward(const void* dy, int64_t dy_pixel, int64_t dy_sample, const void* x, int64_t x_pixel,
                           int64_t x_sample, int dtype, int N, int64_t pixels, int C, int G, const float* gamma,
                           const float* beta, const float* mean, const float* rstd, int act, void* dx, float* dgamma,
                           float* dbeta, void* workspace, size_t workspace_bytes, void* stream) {
    const Shape s{dtype, N, C, G, pixels, true};
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
    if (workspace_bytes < workspace_of(s)) return PP_ERR_BUFFER;
    const size_t xb = (size_t)N * pixels * C * size_of(dtype);
    const bool over_dy = dx == dy && dy_pixel == C && dy_sample == pixels * C;
    if (overlap(x, extent(s, x_pixel, x_sample), dx, xb) ||
        (!over_dy && overlap(dy, extent(s, dy_pixel, dy_sample), dx, xb)))
        return PP_ERR_BUFFER;
    const Plan p = plan_of(s, std::min({align_of(x), align_of(dy), align_of(dx), align_of(C, dtype),
                                          pixels > 1 ? align_of(x_pixel, dtype) : 16,
                                          pixels > 1 ? align_of(dy_pixel, dtype) : 16,
                                          N > 1 ? align_of(x_sample, dtype) : 16,
                                          N > 1 ? align_of(dy_sample, dtype) : 16}));
    NormArgs a = args_of(s, p, x, x_pixel, x_sample, gamma, beta, act, dx, workspace);
    a.dy = dy;
    a.dy_pixel = dy_pixel;
    a.dy_sample = dy_sample;
    a.mean = mean;
    a.rstd = rstd;
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.sums = a.parts + p.parts + (norm_counters(N) + 1) / 2 * 2;
    return done(a, p, s, stream);
}

}  // extern "C"
