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
// of 32 to 512 bytes -- and holds it in shared memory between the sums and the result, the CTAs' sums being
// joined through distributed shared memory, so that every value is read from memory once.
// Streamed form, for units that 8 CTAs do not hold, or not well: one kernel sums (a CTA takes a stretch of
// pixels of a sample, a thread always the same V channels, so that a warp reads whole rows), one joins a
// sample's parts, one has the result.  The second reading comes from L2 where a call's inputs fit there: the
// result takes the samples in the reverse order of the sums.
//
// Measured on a GB300 (a copy moves 6.67 TB/s), inputs in memory, the launches of a call together:
//     forward   32x256x56x56 fp16    27 us, 3.8 TB/s of what it must move   (resident, 4 x 50 KB a unit)
//     forward   32x64x224x224 fp32  195 us, 4.2 TB/s; 6.3 TB/s with the second reading   (streamed)
//     backward  32x512x14x14 fp32    13 us, 3.0 TB/s   (resident, one CTA a unit)
//     backward  32x128x112x112 fp16  91 us, 3.4 TB/s; 5.6 TB/s with the second reading   (streamed)
// The resident form is bound by what its few CTAs on an SM have in flight while some of them wait for their
// clusters and by the arithmetic of SiLU (two operations of the special function unit an element, four
// backward); the streamed one by memory, whose rate falls a little short of a copy's backward.
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
#include <cstdlib>
#include <numeric>

#include "norm.h"
#include "patconv.h"

namespace patconv {

extern template struct NormKernels<float>;
extern template struct NormKernels<__half>;
extern template struct NormKernels<__nv_bfloat16>;

bool norm_starts_early() {
    static const bool on = [] {
        const char* e = std::getenv("PATCONV_PDL");
        return !(e && e[0] == '0');
    }();
    return on;
}

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
    int tiles = 1, chunks = 1;              // streamed: CTAs side by side, stretches down a sample
    int held = 0, depth = 1;                // vectors of each input that a CTA holds; streamed: half a thread's of them
    int cluster = 0, slabs = 1;             // resident: CTAs a unit (0: streamed), slabs
    size_t parts = 0, sums = 0;             // floats of the workspace
};

constexpr int kSMs = 152;
constexpr double kSmShared = 232448;        // bytes of shared memory of an SM
constexpr int64_t kStretch = 131072, kStretchBack = 1048576, kLeast = 8192;        // streamed: bytes of a CTA,
constexpr int kRing = 65536;                                                       // of those it holds at a time
constexpr int64_t kMostHeld = 163840, kSlabLeast = 32, kSlabMost = 512;            // resident: bytes of a CTA, of a slab's pixel

int quarter_of(const Plan& p) { return (p.rows + 3) / 4 * p.cols; }
// resident: bytes of shared memory beside the vectors (the kernels' sums, channels and groups)
int64_t shared_beside(const Shape& s, const Plan& p) {
    const int64_t channels = (int64_t)p.cols * p.V, groups = channels / (s.C / s.G);
    return 8 * ((s.backward ? (int64_t)quarter_of(p) * p.V : (int64_t)p.NS * kNormThreads) + channels + 2 * groups);
}
int places(const Plan& p) { return (p.chunk * p.cols + 7) / 8 * 8; }    // vectors of an input that a CTA holds

// The resident form: of the slabs of whole groups from a 32-byte sector to 512 bytes wide and of the clusters that
// hold them, the one whose estimated time is least.  In us: a CTA takes 4 beside its work (the first copies'
// latency, two barriers of the cluster, the second reading of its parameters); its work is what its share of the
// SM's 44 KB a us moves, or what the arithmetic of its vectors takes, 0.03 a channel of each of its rows of
// vectors (0.06 in vectors of 4 bytes, 0.12 of one channel), and 2.2 times as long where it is alone; and there
// are as many rounds as the SMs need for all CTAs.  Narrow slabs move parts of lines.  Measured, this plan against
// one fixed rule (128 bytes, CTAs of 48 KB): 32x256x56x56 fp16 forward 27 against 35 us, 4x128x112x112 fp16 forward
// 13 against 20, 32x512x14x14 fp32 backward 14 against 25.  Against the streamed form: 32x256x56x56 fp16 forward 27
// against 37, 16x256x28x28 fp32 forward 8 against 20; but 32x128x112x112 fp16 backward, whose slabs would be of 32
// bytes, 136 against 92.
bool resident(const Shape& s, Plan& p) {
    const int es = size_of(s.dtype), bytes = p.V * es, cpg = s.C / s.G, vectors = s.C / p.V, inputs = s.backward ? 2 : 1;
    const int unit = std::lcm(cpg, p.V) / p.V;              // vectors of the least slab of whole groups
    if (unit > kNormThreads || vectors % unit) return false;
    const int steps = vectors / unit;
    double least = 0;
    Plan best;
    for (int m = 1; m <= steps; ++m) {
        const int width = m * unit * bytes;
        if (m * unit > kNormThreads || m * unit * p.V > 1024 || (width > kSlabMost && best.cluster)) break;
        if (steps % m || steps / m > 65535 || (width < kSlabLeast && m < steps)) continue;
        for (int c = 1; c <= 8; c *= 2) {
            const int64_t chunk = (s.pixels + c - 1) / c;
            if (chunk * m * unit * bytes * inputs > kMostHeld) continue;
            Plan q = p;
            q.cols = m * unit;
            q.rows = kNormThreads / q.cols;
            q.slabs = vectors / q.cols;
            q.cluster = c;
            q.chunk = (int)chunk;
            const double held = (double)places(q) * bytes * inputs, rows = (double)((chunk + q.rows - 1) / q.rows);
            const double room = held + shared_beside(s, q);
            if (room > kNormShared) continue;
            const double total = (double)s.N * q.slabs * c, fit = std::min(s.backward ? 3.0 : 4.0, std::floor(kSmShared / (room + 3072)));
            const double rounds = std::ceil(total / (kSMs * fit)), at_once = std::min(fit, std::ceil(total / kSMs));
            const double channel = p.V == 1 ? 0.12 : bytes == 4 ? 0.06 : 0.03, narrow = width >= 48 ? 1.0 : 1.3;
            const double work = rows * p.V * channel * inputs, moved = held / inputs * (inputs + 1) / 44e3;
            const double time = rounds * (4 + 0.1 * c + narrow * std::max({at_once * moved, at_once * work, 2.2 * work}));
            if (!best.cluster || time < least) {
                best = q;
                least = time;
            }
        }
    }
    // streamed: three launches, the inputs twice and the output at 5.5 TB/s
    const double streamed = 20 + (2 * inputs + 1.0) * s.N * s.pixels * s.C * es / 5.5e6;
    if (!best.cluster || least > streamed) return false;
    p = best;
    p.parts = s.backward ? (size_t)s.N * p.cluster * s.C * 2 : 0;
    return true;
}

void set_width(const Shape& s, Plan& p, int V) {
    p.V = V;
    p.NS = s.C / s.G % V ? V : 1;
}

// The streamed form: a row's vectors over the threads of one or more CTAs, stretches of pixels of up to kStretch
// bytes of all inputs (backward kStretchBack), so many that the CTAs fill the SMs a whole number of times (three on
// each, backward two, which have the registers for it), but none below kLeast bytes.  A CTA reads its stretch
// through kRing bytes of shared memory.  Backward a thread has eight channels' parameters to fetch and sums to join,
// which a long stretch pays for: 32x128x112x112 fp16 takes 92 us with up to 1 MB, 99 with 256 KB, 110 with 64 KB
// all held at once, 97 with three CTAs an SM; 48 KB of ring cost 2 us, 96 KB gain nothing.  Forward there is little
// of that, and the stretches of many CTAs at a time are read faster: 32x64x224x224 fp32 takes 195 us with up to
// 128 KB, 198 with 256 KB, 206 with 512 KB, 199 with 48 KB of ring.
void streamed(const Shape& s, Plan& p) {
    const int es = size_of(s.dtype), vectors = s.C / p.V, inputs = s.backward ? 2 : 1;
    p.tiles = (vectors + kNormThreads - 1) / kNormThreads;
    p.cols = (vectors + p.tiles - 1) / p.tiles;
    p.rows = kNormThreads / p.cols;
    const int64_t row = (int64_t)p.cols * p.V * es, side = (int64_t)s.N * p.tiles, full = kSMs * (s.backward ? 2 : 3);
    const int64_t most = std::max<int64_t>(p.rows, (s.backward ? kStretchBack / 2 : kStretch) / row), least = std::max<int64_t>(p.rows, (kLeast + row - 1) / row);
    const int64_t times = std::max<int64_t>(1, (side * ((s.pixels + most - 1) / most) + full - 1) / full);
    const int64_t chunks = std::max<int64_t>(1, times * full / side);
    p.chunk = (int)std::min(s.pixels, std::max(least, (s.pixels + chunks - 1) / chunks));
    p.chunks = (int)((s.pixels + p.chunk - 1) / p.chunk);
    const int vector = p.V * es, mine = (p.chunk + p.rows - 1) / p.rows;
    p.depth = std::min(kRing / 2 / inputs / (vector * kNormThreads), (mine + 1) / 2);
    const size_t sets = s.backward ? s.C : s.C / (p.V / p.NS);
    p.parts = (size_t)s.N * p.chunks * sets * 2;
    p.sums = s.backward ? (size_t)s.N * s.C * 2 + (size_t)s.N * s.G * 2 : 0;
}

// Vectors of 16 bytes a thread where `align`, the common alignment of addresses and strides in bytes, allows it,
// else of 4 bytes or one channel.  Narrower ones than that make a slab of whole groups of odd numbers of channels
// narrow enough for a cluster: 9x312x56x51 fp16 forward in 8 groups takes 14 us so, 27 us streamed.
Plan plan_of(const Shape& s, int align) {
    const int es = size_of(s.dtype), widest = align >= 16 ? 16 / es : std::max(1, std::min(align, 4) / es);
    Plan p;
    for (int V = widest; V && !p.cluster; V = V * es > 4 ? 4 / es : V / 2) {
        set_width(s, p, V);
        resident(s, p);
    }
    if (!p.cluster) {
        set_width(s, p, widest);
        streamed(s, p);
    }
    p.held = p.cluster ? places(p) : (2 * p.depth * p.rows * p.cols + 7) / 8 * 8;
    if (!s.backward) p.sums += (size_t)s.N * s.G * 2;       // mean and rstd that the caller does not want
    return p;
}

// enough for any plan that a call's alignment may lead to
size_t workspace_of(const Shape& s) {
    size_t most = s.backward ? (size_t)s.N * 8 * s.C * 2 : 0;           // resident, in clusters of eight
    for (int align = size_of(s.dtype); align <= 16; align *= 2)
        if ((int64_t)s.C * size_of(s.dtype) % align == 0) {
            Plan p;
            set_width(s, p, align >= 16 ? 16 / size_of(s.dtype) : std::max(1, std::min(align, 4) / size_of(s.dtype)));
            streamed(s, p);
            most = std::max(most, p.parts + p.sums);
        }
    return (most + (s.backward ? 0 : (size_t)s.N * s.G * 2)) * sizeof(float);
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

// whether an input lies as the output does; strides between pixels, or samples, that there is one of do not count
bool dense(const Shape& s, int64_t pixel, int64_t sample) {
    return (s.pixels == 1 || pixel == s.C) && (s.N == 1 || sample == s.pixels * s.C);
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
    return backward ? K::backward(a, p.V, st) : K::forward(a, p.V, p.NS, st);
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
    a.held = p.held;
    a.depth = p.depth;
    a.quarter = quarter_of(p);
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
    return a;
}

int done(const NormArgs& a, const Plan& p, const Shape& s, void* stream) {
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
    const int64_t all[8] = {p.cluster ? 2 : 1, p.V, p.cols, p.chunk, p.held, p.cluster,
                            p.cluster ? (int64_t)N * p.slabs * p.cluster : (int64_t)p.chunks * p.tiles * N, p.NS};
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
    if (!N || !pixels) {                            // all bits set are a NaN: there are no values
        for (float* p : {mean, rstd}) {
            if (off4(p)) return PP_ERR_ALIGN;
            if (p && N && cudaMemsetAsync(p, 0xFF, (size_t)N * G * 4, static_cast<cudaStream_t>(stream)) != cudaSuccess) {
                cudaGetLastError();
                return PP_ERR_CUDA;
            }
        }
        return PP_OK;
    }
    if (const int e = check_input(s, x, x_pixel, x_sample)) return e;
    if (!y || !workspace) return PP_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(y) % size_of(dtype) || off4(gamma) || off4(beta) || off4(mean) || off4(rstd) ||
        reinterpret_cast<uintptr_t>(workspace) % 16)
        return PP_ERR_ALIGN;
    if (workspace_bytes < workspace_of(s)) return PP_ERR_BUFFER;
    const size_t yb = (size_t)N * pixels * C * size_of(dtype);
    // y may be x itself where x is dense: every value is read before it is written
    if (!(x == y && dense(s, x_pixel, x_sample)) && overlap(x, extent(s, x_pixel, x_sample), y, yb))
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
        for (float* p : {dgamma, dbeta})
            if (p && cudaMemsetAsync(p, 0, (size_t)C * 4, st) != cudaSuccess) {
                cudaGetLastError();
                return PP_ERR_CUDA;
            }
        return PP_OK;
    }
    if (const int e = check_input(s, dy, dy_pixel, dy_sample)) return e;
    if (const int e = check_input(s, x, x_pixel, x_sample)) return e;
    if (!mean || !rstd || !dx || !workspace) return PP_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(dx) % size_of(dtype) || reinterpret_cast<uintptr_t>(workspace) % 16)
        return PP_ERR_ALIGN;
    if (workspace_bytes < workspace_of(s)) return PP_ERR_BUFFER;
    const size_t xb = (size_t)N * pixels * C * size_of(dtype);
    const bool over_dy = dx == dy && dense(s, dy_pixel, dy_sample);
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
    a.sums = a.parts + p.parts;
    return done(a, p, s, stream);
}

}  // extern "C"
