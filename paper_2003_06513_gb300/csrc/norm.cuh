// Kernels of norm.cu, for one type of activations each in norm_f32.cu, norm_f16.cu and norm_bf16.cu (three
// translation units, compiled side by side).
//
// The kernels are issue-bound before they are memory-bound if left to scalar code (27 instructions an
// element of a forward pass at 2.2 TB/s): the arithmetic runs on pairs of fp32 values, two to an
// instruction, the activation is chosen outside the loops, and exp and 1 / x are the hardware's
// approximations (2 and 1 ulp) with subnormals flushed.
//
// What a CTA reads goes to shared memory by asynchronous copies: in the resident kernels all of its stretch asked
// for at once, and the sums of the first half taken while the second is under way; in the streamed ones through a
// ring of two halves, one asked for while the other is used.  Held in registers instead (up to 8 vectors a
// thread, one CTA fewer on an SM) the forward pass of 32x256x56x56 fp16 took 38 us, so 27.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstring>
#include <type_traits>

#include "norm.h"
#include "patconv.h"
#include "vec.cuh"

namespace patconv {
namespace {

constexpr int kThreads = kNormThreads;
constexpr int kWarps = kThreads / 32;

// -------------------------------------------------------------------------------- asynchronous copies

// Asynchronous copies into the thread's own places of shared memory, which hold what a thread reads of a
// CTA's stretch: all of it is under way at once, at no cost in registers.  No other thread reads it, so that
// waiting for the thread's own copies is all that is needed.
template <typename T, int V>
__device__ __forceinline__ void copy_async(Vec<T, V>* to, const T* from) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(to);
    static_assert(sizeof(T) * V == 16 || sizeof(T) * V == 4, "sizes that the copies have");
    if constexpr (sizeof(T) * V == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(from) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(d), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// -------------------------------------------------------------------------------- joining moments

struct Moments {
    float n, mean, m2;
};
__device__ __forceinline__ Moments join(const Moments& a, const Moments& b) {
    if (a.n == 0.0f) return b;
    if (b.n == 0.0f) return a;
    const float n = a.n + b.n, f = b.n * approx_rcp(n), d = b.mean - a.mean;
    return {n, fmaf(d, f, a.mean), a.m2 + fmaf(d * d, a.n * f, b.m2)};
}
// over the lanes' aligned sets of L, into the first of each
template <int L>
__device__ __forceinline__ Moments join_lanes(Moments m) {
#pragma unroll
    for (int o = L / 2; o; o >>= 1) {
        const Moments b{__shfl_down_sync(0xffffffffu, m.n, o), __shfl_down_sync(0xffffffffu, m.mean, o),
                        __shfl_down_sync(0xffffffffu, m.m2, o)};
        m = join(m, b);
    }
    return m;
}
template <int L>
__device__ __forceinline__ float2 sum_lanes(float2 s) {
#pragma unroll
    for (int o = L / 2; o; o >>= 1)
        s = add(s, make_float2(__shfl_down_sync(0xffffffffu, s.x, o), __shfl_down_sync(0xffffffffu, s.y, o)));
    return s;
}

// f(k, how many) for k from first to end - 1, U at a time while there are as many, then one at a time
template <int U, typename F>
__device__ __forceinline__ void by_batches(int first, int end, F&& f) {
#pragma unroll 1
    for (; first + U <= end; first += U) f(first, std::integral_constant<int, U>());
#pragma unroll 1
    for (; first < end; ++first) f(first, std::integral_constant<int, 1>());
}
// What a thread holds of one input: vectors of its rows, the first half of them in a group of copies of its own.
template <typename T, int V>
struct Held {
    Vec<T, V>* mine;
    int step;
    // one place a vector of the CTA's pixels; the input's places begin at `from`
    __device__ __forceinline__ Held(const NormArgs& a, void* smem, int from = 0)
        : mine(static_cast<Vec<T, V>*>(smem) + from + threadIdx.x), step(a.rows * a.cols) {}
    // asks for vectors first to end - 1, the first of them at p, which goes on to the next
    __device__ __forceinline__ void copy(const T*& p, int64_t stride, int first, int end) const {
        if constexpr (sizeof(T) * V >= 4) {
#pragma unroll 2
            for (int k = first; k < end; ++k, p += stride) copy_async(mine + k * step, p);
        } else {                      // there is no copy of two bytes: eight readings under way at a time
            by_batches<8>(first, end, [&](int k, auto batch) {
                constexpr int K = decltype(batch)::value;
                Vec<T, V> v[K];
#pragma unroll
                for (int u = 0; u < K; ++u, p += stride) v[u] = load<T, V>(p);
#pragma unroll
                for (int u = 0; u < K; ++u) mine[(k + u) * step] = v[u];
            });
        }
    }
    __device__ __forceinline__ const Vec<T, V>& operator[](int k) const { return mine[k * step]; }
    // vector k in the place of vector k - shift
    __device__ __forceinline__ Held from(int shift) const {
        Held h = *this;
        h.mine -= shift * step;
        return h;
    }
};
// f(first, end) for the first half, then for the rest, each as soon as its copies have come
template <typename F>
__device__ __forceinline__ void as_they_come(int count, F&& f) {
    const int half = (count + 1) / 2;
    copies_wait<1>();
    f(0, half);
    copies_wait<0>();
    f(half, count);
}

// A thread's `count` vectors through places for 2 x depth of them, `depth` at a time: use(shift, first, end) gets them
// as soon as their copies have come, with vector k in place k - shift, and copy(shift, first, end) asks for those
// that take the places of the ones used.
template <typename Copy, typename Use>
__device__ __forceinline__ void flow(int count, int depth, Copy&& copy, Use&& use) {
    copy(0, 0, min(depth, count));
    copies_end();
    copy(0, depth, min(2 * depth, count));
    copies_end();
    int shift = 0;
    bool second = false;
#pragma unroll 1
    for (int k = 0; k < count; k += depth) {
        copies_wait<1>();
        use(shift, k, min(k + depth, count));
        copy(shift + 2 * depth, k + 2 * depth, min(k + 3 * depth, count));
        copies_end();
        shift += second ? 2 * depth : 0;
        second = !second;
    }
}

// A thread's moments of NS sets of S = V / NS adjacent channels, each within one group.
template <typename T, int V, int NS>
struct Sets {
    static constexpr int P = NS == 1 ? 1 : kPairs<V>;            // pairs of sets (one set: its first)
    float2 mean[P] = {}, m2[P] = {};
    float n = 0.0f;                                              // pixels so far

    // K vectors, the first k of them given, taken by their distance from the first: a constant's mean and
    // variance are exact, and the sum of squares is at most k S + 1 times what is left of it
    template <int K>
    __device__ __forceinline__ void take(const Vec<T, V> (&v)[K], int k) {
        if (k <= 0) return;
        const float total = n + (float)k, f = n == 0.0f ? 1.0f : (float)k * approx_rcp(total), w = n * f;
        if constexpr (NS == 1) {
            const float x0 = widen(v[0].v[0]);
            const float2 shift = both(-x0);
            float2 s[2] = {}, q[2] = {};
#pragma unroll
            for (int u = 0; u < K; ++u)
                if (u < k) {
#pragma unroll
                    for (int i = 0; i < kPairs<V>; ++i) {
                        const float2 d = add(pair(v[u], i), shift);
                        s[u % 2] = add(s[u % 2], d);
                        q[u % 2] = fma(d, d, q[u % 2]);
                    }
                }
            const float2 ss = add(s[0], s[1]), qq = add(q[0], q[1]);
            const float sum = V == 1 ? ss.x : ss.x + ss.y, square = V == 1 ? qq.x : qq.x + qq.y;
            const float mu = sum * approx_rcp((float)(k * V));
            merge1(fmaf(-mu, sum, square), mu + x0, f, w * V);
        } else {
            const float inv = approx_rcp((float)k);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float2 x0 = pair(v[0], i), shift = neg(x0);
                float2 s = {}, q = {};
#pragma unroll
                for (int u = 1; u < K; ++u)
                    if (u < k) {
                        const float2 d = add(pair(v[u], i), shift);
                        s = add(s, d);
                        q = fma(d, d, q);
                    }
                const float2 mu = mul(s, both(inv));
                q = fma(neg(mu), s, q);
                const float2 d = add(add(mu, x0), neg(mean[i]));
                mean[i] = fma(d, both(f), mean[i]);
                m2[i] = add(m2[i], fma(mul(d, d), both(w), make_float2(positive(q.x), positive(q.y))));
            }
        }
        n = total;
    }
    template <int U>
    __device__ __forceinline__ void take_all(const Held<T, V>& held, int first, int end) {
        by_batches<U>(first, end, [&](int k, auto batch) {
            constexpr int K = decltype(batch)::value;
            Vec<T, V> v[K];
#pragma unroll
            for (int u = 0; u < K; ++u) v[u] = held[k + u];
            take(v, K);
        });
    }
    __device__ static __forceinline__ float positive(float q) { return q < 0.0f ? 0.0f : q; }   // NaN stays
    __device__ __forceinline__ void merge1(float q, float mu, float f, float w) {
        const float d = mu - mean[0].x;
        mean[0].x = fmaf(d, f, mean[0].x);
        m2[0].x += fmaf(d * d, w, positive(q));
    }
    // [set][thread] in shared memory: mean, m2
    __device__ __forceinline__ void put(float2* s) const {
#pragma unroll
        for (int j = 0; j < NS; ++j)
            s[j * kThreads + threadIdx.x] = j % 2 ? make_float2(mean[j / 2].y, m2[j / 2].y) : make_float2(mean[j / 2].x, m2[j / 2].x);
    }
};

// -------------------------------------------------------------------------------- activations

constexpr float kLog2e = 1.4426950408889634f;

template <int ACT>
__device__ __forceinline__ float activated1(float z) {
    if constexpr (ACT == PP_ACT_RELU) {
        float r;
        asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(z));
        return r;
    }
    return z;
}
template <int ACT>
__device__ __forceinline__ float2 activated(float2 z) {
    if constexpr (ACT == PP_ACT_SILU) {
        const float2 e = mul(z, both(-kLog2e));
        const float2 d = add(make_float2(approx_exp2(e.x), approx_exp2(e.y)), both(1.0f));
        return mul(z, make_float2(approx_rcp(d.x), approx_rcp(d.y)));
    }
    return make_float2(activated1<ACT>(z.x), activated1<ACT>(z.y));
}
// dy act'(z)
template <int ACT>
__device__ __forceinline__ float2 through(float2 dy, float2 z) {
    if constexpr (ACT == PP_ACT_RELU) return make_float2(z.x > 0.0f ? dy.x : 0.0f, z.y > 0.0f ? dy.y : 0.0f);
    if constexpr (ACT == PP_ACT_SILU) {
        const float2 e = mul(z, both(-kLog2e));
        const float2 d = add(make_float2(approx_exp2(e.x), approx_exp2(e.y)), both(1.0f));
        const float2 s = make_float2(approx_rcp(d.x), approx_rcp(d.y));
        // s (1 + z (1 - s))
        return mul(mul(dy, s), fma(z, fma(s, both(-1.0f), both(1.0f)), both(1.0f)));
    }
    return dy;
}
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {       // the same for all threads
    if (act == PP_ACT_RELU)
        f(std::integral_constant<int, PP_ACT_RELU>());
    else if (act == PP_ACT_SILU)
        f(std::integral_constant<int, PP_ACT_SILU>());
    else
        f(std::integral_constant<int, PP_ACT_NONE>());
}

// -------------------------------------------------------------------------------- a thread's channels

// A channel's group by a multiplication (cpg_mul = ceil(2^32 / cpg), exact for C up to 2^20), the next
// channels' by counting.
struct GroupOf {
    int g, r, cpg;
    __device__ __forceinline__ GroupOf(const NormArgs& a, int c) : cpg(a.cpg) {
        g = a.cpg == 1 ? c : (int)__umulhi((uint32_t)c, a.cpg_mul);
        if (g * cpg > c) --g;
        r = c - g * cpg;
    }
    __device__ __forceinline__ void next() {
        if (++r == cpg) {
            r = 0;
            ++g;
        }
    }
};

// mean, rstd gamma and beta of the V channels from c of sample n
template <int V>
struct Forward {
    float2 mean[kPairs<V>], scale[kPairs<V>], shift[kPairs<V>];
    template <typename Stat>
    __device__ __forceinline__ Forward(const NormArgs& a, int c, Stat&& stat)
        : Forward(a, c, stat, a.gamma ? a.gamma + c : nullptr, a.beta ? a.beta + c : nullptr) {}
    // gamma, beta: of the V channels, or NULL
    template <typename Stat>
    __device__ __forceinline__ Forward(const NormArgs& a, int c, Stat&& stat, const float* gamma, const float* beta) {
        float m[2] = {}, s[2] = {}, b[2] = {};
        GroupOf at(a, c);
#pragma unroll
        for (int i = 0; i < V; ++i, at.next()) {
            const float2 st = stat(at.g);
            m[i % 2] = st.x;
            s[i % 2] = st.y * (gamma ? gamma[i] : 1.0f);
            b[i % 2] = beta ? beta[i] : 0.0f;
            mean[i / 2] = make_float2(-m[0], -m[1]);
            scale[i / 2] = make_float2(s[0], s[1]);
            shift[i / 2] = make_float2(b[0], b[1]);
        }
    }
    template <int ACT, typename T>
    __device__ __forceinline__ Vec<T, V> apply(Vec<T, V> v) const {
#pragma unroll
        for (int i = 0; i < kPairs<V>; ++i)
            set_pair(v, i, activated<ACT>(fma(add(pair(v, i), mean[i]), scale[i], shift[i])));
        return v;
    }
    // y: where vector `first` of the result goes; then where `end` would
    template <int ACT, typename T>
    __device__ __forceinline__ void write(const NormArgs& a, const Held<T, V>& held, int first, int end, T*& y) const {
        const int64_t step = (int64_t)a.rows * a.C;
        by_batches<2>(first, end, [&](int k, auto batch) {
#pragma unroll
            for (int u = 0; u < decltype(batch)::value; ++u, y += step) store<T, V>(y, apply<ACT>(held[k + u]));
        });
    }
};

// With d = x - mean and s = rstd gamma: z = s d + beta, and
//     dx = rstd (gamma dz - A / M - xh B / M) = s dz + p + q d,  p = -rstd A / M,  q = -rstd^2 B / M,
// A / M and B' / M = rstd B / M coming from sums of dz and of dz d.  A group of one value (M = 1) has dx = 0.
template <int V>
struct Backward {
    float2 mean[kPairs<V>], scale[kPairs<V>], shift[kPairs<V>];
    __device__ __forceinline__ Backward(const NormArgs& a, int n, int c) {
        float m[2] = {}, s[2] = {}, b[2] = {};
        const float *mean_n = a.mean + (int64_t)n * a.G, *rstd_n = a.rstd + (int64_t)n * a.G;
        GroupOf at(a, c);
#pragma unroll
        for (int i = 0; i < V; ++i, at.next()) {
            m[i % 2] = -__ldg(mean_n + at.g);
            s[i % 2] = __ldg(rstd_n + at.g) * (a.gamma ? __ldg(a.gamma + c + i) : 1.0f);
            b[i % 2] = a.beta ? __ldg(a.beta + c + i) : 0.0f;
            mean[i / 2] = make_float2(m[0], m[1]);
            scale[i / 2] = make_float2(s[0], s[1]);
            shift[i / 2] = make_float2(b[0], b[1]);
        }
    }
    // sums of dz and of dz d
    template <int ACT, typename T>
    __device__ __forceinline__ void sum(const Vec<T, V>& x, const Vec<T, V>& dy, float2 (&sb)[kPairs<V>], float2 (&sg)[kPairs<V>]) const {
#pragma unroll
        for (int i = 0; i < kPairs<V>; ++i) {
            const float2 d = add(pair(x, i), mean[i]), dz = through<ACT>(pair(dy, i), fma(d, scale[i], shift[i]));
            sb[i] = add(sb[i], dz);
            sg[i] = fma(dz, d, sg[i]);
        }
    }
    template <int ACT, typename T>
    __device__ __forceinline__ void sum_all(const Held<T, V>& x, const Held<T, V>& dy, int first, int end,
                                            float2 (&sb)[kPairs<V>], float2 (&sg)[kPairs<V>]) const {
#pragma unroll 1
        for (int k = first; k < end; ++k) sum<ACT>(x[k], dy[k], sb, sg);
    }
    // pq: p, p', q, q' of a pair
    template <int ACT, typename T>
    __device__ __forceinline__ Vec<T, V> apply(Vec<T, V> x, const Vec<T, V>& dy, const float4 (&pq)[kPairs<V>], float one) const {
#pragma unroll
        for (int i = 0; i < kPairs<V>; ++i) {
            const float2 d = add(pair(x, i), mean[i]), dz = through<ACT>(pair(dy, i), fma(d, scale[i], shift[i]));
            const float2 rest = fma(d, make_float2(pq[i].z, pq[i].w), make_float2(pq[i].x, pq[i].y));
            set_pair(x, i, fma(mul(scale[i], both(one)), dz, rest));
        }
        return x;
    }
    // dx: where vector `first` of the result goes; then where `end` would
    template <int ACT, typename T>
    __device__ __forceinline__ void write(const NormArgs& a, const Held<T, V>& x, const Held<T, V>& dy, int first, int end, T*& dx,
                                          const float4 (&pq)[kPairs<V>]) const {
        const int64_t step = (int64_t)a.rows * a.C;
        const float one = a.pixels * a.cpg == 1 ? 0.0f : 1.0f;
#pragma unroll 1
        for (int k = first; k < end; ++k, dx += step) store<T, V>(dx, apply<ACT>(x[k], dy[k], pq, one));
    }
};
// p and q of a thread's groups by pairs of channels; stat(g) gives them
template <int V, typename Stat>
__device__ __forceinline__ void pair_stats(float4 (&out)[kPairs<V>], const NormArgs& a, int c, Stat&& stat) {
    float p[2] = {}, q[2] = {};
    GroupOf at(a, c);
#pragma unroll
    for (int i = 0; i < V; ++i, at.next()) {
        const float2 s = stat(at.g);
        p[i % 2] = s.x;
        q[i % 2] = s.y;
        out[i / 2] = make_float4(p[0], p[1], q[0], q[1]);
    }
}
// p and q of a group from its sums of gamma dz and of gamma dz d.  q's factors rstd are taken one at a time: the mean
// of gamma dz d has the size of a value's distance, B / M that of dz, and rstd^3 by itself would leave fp32's range
// for spreads above 1e12 or below 1e-13.
__device__ __forceinline__ float2 group_pq(const NormArgs& a, float2 sums, float rstd) {
    const float inv = 1.0f / ((float)a.pixels * a.cpg), b = rstd * (sums.y * inv);
    return a.pixels * a.cpg == 1 ? make_float2(0.0f, 0.0f) : make_float2(-rstd * (sums.x * inv), -rstd * (rstd * b));
}
// The threads' sums of dz and of dz d by a quarter of their rows: s[channel][row of the quarter][column], the
// rows of the other quarters added in turn.  A quarter of the room is a CTA more on an SM.
template <int V>
__device__ __forceinline__ void put_sums(const NormArgs& a, int row, int col, float2* s, const float2 (&sb)[kPairs<V>], const float2 (&sg)[kPairs<V>]) {
    const int quarter = (a.rows + 3) / 4, size = quarter * a.cols;
    for (int from = 0; from < a.rows; from += quarter) {
        if (row >= from && row < from + quarter && row < a.rows) {
            float2* to = s + (row - from) * a.cols + col;
#pragma unroll
            for (int i = 0; i < V; ++i, to += size) {
                const float2 v = i % 2 ? make_float2(sb[i / 2].y, sg[i / 2].y) : make_float2(sb[i / 2].x, sg[i / 2].x);
                *to = from ? add(*to, v) : v;
            }
        }
        __syncthreads();
    }
}
// A channel's sum over the quarter's rows, in the first of eight lanes.
__device__ __forceinline__ float2 sum_rows(const NormArgs& a, const float2* s, int channel, int col) {
    const int quarter = (a.rows + 3) / 4;
    s += channel * quarter * a.cols + col;
    float2 sum = {};
    for (int r = threadIdx.x % 8; r < quarter; r += 8) sum = add(sum, s[r * a.cols]);
    return sum_lanes<8>(sum);
}

// Between the kernels of one call: a kernel lets the next one start when all of its own CTAs have, and the next one
// waits for the end of all before it where it reads what they write.  The first kernel of a call starts after
// everything before it in the stream, so that the call's inputs are there for any of them.  Against launches that
// wait for one another's end: streamed forward 32x64x224x224 fp32 200 -> 195 us, streamed backward 32x128x112x112
// fp16 113 -> 109 us (before its ring), resident backward 5x150x61x45 bf16 16 -> 14 us.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// -------------------------------------------------------------------------------- streamed kernels

// Three launches: sums, a CTA a stretch of one sample's pixels; the parts of each sample joined; the result.
// What the result reads last of the sums' inputs it reads first, from the L2 cache.

struct Thread {                       // of a CTA: its column and its row
    int col, row;
    __device__ __forceinline__ explicit Thread(const NormArgs& a) {
        row = a.cols == 1 ? threadIdx.x : (int)__umulhi(threadIdx.x, a.cols_mul);
        col = threadIdx.x - row * a.cols;
    }
};
struct Stretch {                      // chunk blockIdx.x and tile blockIdx.y of sample n
    int n, c, col, row, count, mine;  // count: its pixels; mine: this thread's, from row on; c: its channels
    int64_t begin;
    __device__ __forceinline__ Stretch(const NormArgs& a, int V, int sample) : n(sample) {
        const Thread th(a);
        col = th.col;
        row = th.row;
        c = (blockIdx.y * a.cols + col) * V;
        begin = (int64_t)blockIdx.x * a.chunk;
        count = (int)min((int64_t)a.chunk, a.pixels - begin);
        mine = row < a.rows && c < a.C && row < count ? (count - row + a.rows - 1) / a.rows : 0;
    }
};

// parts[n][chunk][set] = mean, m2 of a stretch
template <typename T, int V, int NS>
__global__ void __launch_bounds__(kThreads, 3) norm_sums(NormArgs a) {
    constexpr int S = V / NS, U = 4;
    extern __shared__ uint4 smem4[];
    __shared__ float2 s_sets[NS * kThreads];
    __shared__ int s_mine[kThreads];
    const Stretch at(a, V, blockIdx.z);
    let_next_start();
    {
        const T* x = static_cast<const T*>(a.x) + at.n * a.x_sample + (at.begin + at.row) * a.x_pixel + at.c;
        const Held<T, V> v(a, smem4);
        Sets<T, V, NS> m;
        flow(at.mine, a.depth, [&](int shift, int first, int end) { v.from(shift).copy(x, a.rows * a.x_pixel, first, end); },
             [&](int shift, int first, int end) { m.template take_all<U>(v.from(shift), first, end); });
        m.put(s_sets);
    }
    s_mine[threadIdx.x] = at.mine * S;
    __syncthreads();
    // eight lanes a set, over the rows
    const int sets = a.C / S, here = min(a.cols, a.C / V - (int)blockIdx.y * a.cols) * NS, lane = threadIdx.x % 8;
    float2* parts = reinterpret_cast<float2*>(a.parts) + ((int64_t)at.n * a.chunks + blockIdx.x) * sets + blockIdx.y * a.cols * NS;
    for (int j0 = threadIdx.x / 8; j0 < (here + 3) / 4 * 4; j0 += kThreads / 8) {
        const int j = min(j0, here - 1), col = j / NS, k = j % NS;
        Moments m{0.0f, 0.0f, 0.0f};
        for (int r = lane; r < a.rows; r += 8) {
            const int t = r * a.cols + col;
            const float2 s = s_sets[k * kThreads + t];
            m = join(m, {(float)s_mine[t], s.x, s.y});
        }
        m = join_lanes<8>(m);
        if (lane == 0 && j0 < here) parts[j] = make_float2(m.mean, m.m2);
    }
}

// A group's mean and rstd from its sets' parts, a CTA a group of a sample; S channels a set.
__global__ void __launch_bounds__(kThreads) norm_join(NormArgs a, int S) {
    __shared__ Moments s_warp[kWarps];
    let_next_start();
    wait_for_previous();
    const int g = blockIdx.x, n = blockIdx.y, sets = a.C / S, total = a.chunks * a.spg;
    const float2* parts = reinterpret_cast<const float2*>(a.parts) + (int64_t)n * a.chunks * sets + g * a.spg;
    Moments m{0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int e = threadIdx.x; e < total; e += kThreads) {
        const int k = a.spg == 1 ? e : e / a.spg;
        const float2 p = parts[(int64_t)k * sets + (e - k * a.spg)];
        const int64_t left = a.pixels - (int64_t)k * a.chunk;
        m = join(m, {(float)(left < a.chunk ? left : a.chunk) * S, p.x, p.y});
    }
    m = join_lanes<32>(m);
    if (threadIdx.x % 32 == 0) s_warp[threadIdx.x / 32] = m;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    m = threadIdx.x < kWarps ? s_warp[threadIdx.x] : Moments{0.0f, 0.0f, 0.0f};
    m = join_lanes<kWarps>(m);
    if (threadIdx.x) return;
    const float var = m.m2 / ((float)a.pixels * a.cpg);
    a.mean_out[(int64_t)n * a.G + g] = m.mean;
    a.rstd_out[(int64_t)n * a.G + g] = 1.0f / sqrtf(var + a.eps);
}

template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 3) norm_result(NormArgs a) {
    extern __shared__ uint4 smem4[];
    const Stretch at(a, V, a.N - 1 - blockIdx.z);
    if (!at.mine) return;
    const T* x = static_cast<const T*>(a.x) + at.n * a.x_sample + (at.begin + at.row) * a.x_pixel + at.c;
    const Held<T, V> v(a, smem4);
    T* y = static_cast<T*>(a.out) + ((int64_t)at.n * a.pixels + at.begin + at.row) * a.C + at.c;
    wait_for_previous();
    const float *mean = a.mean_out + (int64_t)at.n * a.G, *rstd = a.rstd_out + (int64_t)at.n * a.G;
    const Forward<V> f(a, at.c, [&](int g) { return make_float2(mean[g], rstd[g]); });
    with_act(a.act, [&](auto act) {
        flow(at.mine, a.depth, [&](int shift, int first, int end) { v.from(shift).copy(x, a.rows * a.x_pixel, first, end); },
             [&](int shift, int first, int end) { f.template write<decltype(act)::value>(a, v.from(shift), first, end, y); });
    });
}

// a thread's vectors of x and dy: from pixel `pixel` of sample n on
template <typename T, int V>
struct Inputs {
    const T *x, *dy;                  // the next to ask for
    Held<T, V> hx, hd;
    __device__ __forceinline__ Inputs(const NormArgs& a, void* smem, int n, int64_t pixel, int c)
        : x(static_cast<const T*>(a.x) + n * a.x_sample + pixel * a.x_pixel + c),
          dy(static_cast<const T*>(a.dy) + n * a.dy_sample + pixel * a.dy_pixel + c),
          hx(a, smem),
          hd(a, smem, a.held) {}
    __device__ __forceinline__ void copy(const NormArgs& a, int shift, int first, int end) {
        hx.from(shift).copy(x, a.rows * a.x_pixel, first, end);
        hd.from(shift).copy(dy, a.rows * a.dy_pixel, first, end);
    }
};

// parts[n][chunk][c] = sums of dz and of dz d of a stretch
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 2) norm_back_sums(NormArgs a) {
    extern __shared__ uint4 smem4[];
    float2* s_sums = reinterpret_cast<float2*>(static_cast<Vec<T, V>*>(static_cast<void*>(smem4)) + 2 * a.held);
    const Stretch at(a, V, blockIdx.z);
    let_next_start();
    float2 sb[kPairs<V>] = {}, sg[kPairs<V>] = {};
    if (at.mine) {
        Inputs<T, V> in(a, smem4, at.n, at.begin + at.row, at.c);
        const Backward<V> f(a, at.n, at.c);
        with_act(a.act, [&](auto act) {
            flow(at.mine, a.depth, [&](int shift, int first, int end) { in.copy(a, shift, first, end); },
                 [&](int shift, int first, int end) {
                     f.template sum_all<decltype(act)::value>(in.hx.from(shift), in.hd.from(shift), first, end, sb, sg);
                 });
        });
    }
    put_sums<V>(a, at.row, at.col, s_sums, sb, sg);
    const int here = min(a.cols * V, a.C - (int)blockIdx.y * a.cols * V), lane = threadIdx.x % 8;
    float2* parts = reinterpret_cast<float2*>(a.parts) + ((int64_t)at.n * a.chunks + blockIdx.x) * a.C + blockIdx.y * a.cols * V;
    for (int j0 = threadIdx.x / 8; j0 < (here + 3) / 4 * 4; j0 += kThreads / 8) {
        const int j = min(j0, here - 1), col = j / V, i = j % V;
        const float2 s = sum_rows(a, s_sums, i, col);
        if (lane == 0 && j0 < here) parts[j] = s;
    }
}

// A CTA a group of a sample: sums[n][c] = (sum of dz, of dz xh), then [n][g] = p and q.  Its threads take 2^bits
// channels (all of the group's, up to 256) and the rest of them the parts in turn.
__global__ void __launch_bounds__(kThreads) norm_back_join(NormArgs a, int bits) {
    __shared__ float2 s_sum[kThreads], s_warp[kWarps];
    let_next_start();
    wait_for_previous();
    const int g = blockIdx.x, n = blockIdx.y, wide = 1 << bits, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const float rstd = a.rstd[(int64_t)n * a.G + g];
    const float2* parts = reinterpret_cast<const float2*>(a.parts) + (int64_t)n * a.chunks * a.C + g * a.cpg;
    float2 *channel = reinterpret_cast<float2*>(a.sums), *group = channel + (int64_t)a.N * a.C, all = {};
    for (int i0 = 0; i0 < a.cpg; i0 += wide) {
        const int i = i0 + (threadIdx.x & (wide - 1));
        float2 s = {};
        if (i < a.cpg)
#pragma unroll 4
            for (int k = threadIdx.x >> bits; k < a.chunks; k += kThreads >> bits) s = add(s, parts[(int64_t)k * a.C + i]);
        for (int o = 16; o >= wide; o >>= 1)                    // the warp's sums of a channel
            s = add(s, make_float2(__shfl_down_sync(0xffffffffu, s.x, o), __shfl_down_sync(0xffffffffu, s.y, o)));
        s_sum[threadIdx.x] = s;
        __syncthreads();
        const int step = max(1, wide / 32);                     // warps that hold the same channels are as far apart
        if (threadIdx.x < wide && i < a.cpg) {
            for (int w = warp + step; w < kWarps; w += step) s = add(s, s_sum[w * 32 + lane]);
            channel[(int64_t)n * a.C + g * a.cpg + i] = make_float2(s.x, rstd * s.y);
            all = fma(both(a.gamma ? a.gamma[g * a.cpg + i] : 1.0f), s, all);
        }
        __syncthreads();
    }
    all = sum_lanes<32>(all);
    if (lane == 0) s_warp[warp] = all;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < kWarps; ++w) all = add(all, s_warp[w]);
    group[(int64_t)n * a.G + g] = group_pq(a, all, rstd);
}

// dgamma and dbeta, a warp 32 channels and the CTA's warps the parts [part][C] in turn, in their order
__device__ __forceinline__ void norm_back_params(const NormArgs& a, const float2* from, int parts, int block) {
    __shared__ float2 s[kThreads];
    const int c = block * 32 + threadIdx.x % 32;
    float2 sum = {};
    if (c < a.C) {
#pragma unroll 8
        for (int k = threadIdx.x / 32; k < parts; k += kWarps) sum = add(sum, from[(int64_t)k * a.C + c]);
    }
    s[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x >= 32 || c >= a.C) return;
    for (int w = 1; w < kWarps; ++w) sum = add(sum, s[w * 32 + threadIdx.x]);
    if (a.dbeta) a.dbeta[c] = sum.x;
    if (a.dgamma) a.dgamma[c] = sum.y;
}

// dx, and in the CTAs of blockIdx.z = 0 the sums over the samples
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 2) norm_back_result(NormArgs a) {
    extern __shared__ uint4 smem4[];
    const float2 *channel = reinterpret_cast<const float2*>(a.sums), *group = channel + (int64_t)a.N * a.C;
    if (blockIdx.z == 0) {
        wait_for_previous();
        if (a.dgamma || a.dbeta)
            for (int block = blockIdx.y * gridDim.x + blockIdx.x; block * 32 < a.C; block += gridDim.x * gridDim.y) {
                norm_back_params(a, channel, a.N, block);
                __syncthreads();
            }
        return;
    }
    const Stretch at(a, V, a.N - blockIdx.z);
    if (!at.mine) return;
    Inputs<T, V> in(a, smem4, at.n, at.begin + at.row, at.c);
    const Backward<V> f(a, at.n, at.c);
    wait_for_previous();
    float4 pq[kPairs<V>];
    pair_stats<V>(pq, a, at.c, [&](int g) { return group[(int64_t)at.n * a.G + g]; });
    T* dx = static_cast<T*>(a.out) + ((int64_t)at.n * a.pixels + at.begin + at.row) * a.C + at.c;
    with_act(a.act, [&](auto act) {
        flow(at.mine, a.depth, [&](int shift, int first, int end) { in.copy(a, shift, first, end); },
             [&](int shift, int first, int end) {
                 f.template write<decltype(act)::value>(a, in.hx.from(shift), in.hd.from(shift), first, end, dx, pq);
             });
    });
}

// -------------------------------------------------------------------------------- resident kernels

namespace cg = cooperative_groups;

// A unit of the resident kernels is a sample's slab: `cols` vectors of every pixel, whole groups.  The CTAs
// of a cluster take a stretch of its pixels each and hold it in shared memory between the sums and the
// result, so that every value is read from memory once.
template <int V>
struct Unit {
    int rank, slab, n, col, row, c, count, mine;     // count: the CTA's pixels; mine: this thread's
    int64_t begin;
    __device__ __forceinline__ explicit Unit(const NormArgs& a) {
        rank = blockIdx.x;
        slab = blockIdx.y;
        n = blockIdx.z;
        const Thread th(a);
        col = th.col;
        row = th.row;
        c = (slab * a.cols + col) * V;
        begin = (int64_t)rank * a.chunk;
        count = pixels(a, rank);
        // rows_mul is exact for a resident CTA's few thousand pixels
        mine = row < a.rows && row < count ? (a.rows == 1 ? count : (int)__umulhi(count - row + a.rows - 1, a.rows_mul)) : 0;
    }
    __device__ static __forceinline__ int pixels(const NormArgs& a, int rank) {
        const int64_t left = a.pixels - (int64_t)rank * a.chunk;
        return left < 0 ? 0 : left < a.chunk ? (int)left : a.chunk;
    }
};

template <typename T, int V, int NS>
__global__ void __launch_bounds__(kThreads, 4) norm_resident(NormArgs a) {
    constexpr int S = V / NS;
    extern __shared__ uint4 smem4[];
    float2* s_sets = reinterpret_cast<float2*>(static_cast<Vec<T, V>*>(static_cast<void*>(smem4)) + a.held);
    float2 *s_part = s_sets + NS * kThreads, *s_stat = s_part + a.groups;   // the CTA's groups: mean, m2; the cluster's: mean, rstd
    float* s_affine = reinterpret_cast<float*>(s_stat + a.groups);          // the slab's gamma, then beta
    __shared__ int s_mine[kThreads];
    const Unit<V> at(a);
    const int lane = threadIdx.x % 32, width = a.cols * V;
    const T* x = static_cast<const T*>(a.x) + at.n * a.x_sample + (at.begin + at.row) * a.x_pixel + at.c;
    const Held<T, V> v(a, smem4);
    {
        const int half = (at.mine + 1) / 2;
        v.copy(x, a.rows * a.x_pixel, 0, half);
        copies_end();
        v.copy(x, a.rows * a.x_pixel, half, at.mine);
        copies_end();
        for (int j = threadIdx.x; j < width; j += kThreads) {
            s_affine[j] = a.gamma ? a.gamma[at.slab * width + j] : 1.0f;
            s_affine[width + j] = a.beta ? a.beta[at.slab * width + j] : 0.0f;
        }
        Sets<T, V, NS> m;
        as_they_come(at.mine, [&](int first, int end) { m.template take_all<4>(v, first, end); });
        m.put(s_sets);
    }
    s_mine[threadIdx.x] = at.mine * S;
    __syncthreads();
    for (int g = threadIdx.x / 32; g < a.groups; g += kWarps) {             // a warp a group
        Moments m{0.0f, 0.0f, 0.0f};
        for (int e = lane; e < a.rows * a.spg; e += 32) {
            const int r = a.spg == 1 ? e : (int)__umulhi(e, a.spg_mul);
            const int set = g * a.spg + e - r * a.spg, t = r * a.cols + set / NS;
            const float2 s = s_sets[set % NS * kThreads + t];
            m = join(m, {(float)s_mine[t], s.x, s.y});
        }
        m = join_lanes<32>(m);
        if (lane == 0) s_part[g] = make_float2(m.mean, m.m2);
    }
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    for (int g = threadIdx.x; g < a.groups; g += kThreads) {
        Moments m{0.0f, 0.0f, 0.0f};
        for (int r = 0; r < a.cluster; ++r) {
            const float2 p = *cluster.map_shared_rank(s_part + g, r);
            m = join(m, {(float)Unit<V>::pixels(a, r) * a.cpg, p.x, p.y});
        }
        const float var = m.m2 / ((float)a.pixels * a.cpg), rstd = 1.0f / sqrtf(var + a.eps);
        s_stat[g] = make_float2(m.mean, rstd);
        if (at.rank == 0) {
            const int64_t i = (int64_t)at.n * a.G + at.slab * a.groups + g;
            a.mean_out[i] = m.mean;
            a.rstd_out[i] = rstd;
        }
    }
    __syncthreads();
    cluster.barrier_arrive();                                     // the others' parts are read
    if (at.mine) {
        const int first = at.slab * a.groups;
        const Forward<V> f(a, at.c, [&](int g) { return s_stat[g - first]; }, s_affine + at.col * V, s_affine + width + at.col * V);
        T* y = static_cast<T*>(a.out) + ((int64_t)at.n * a.pixels + at.begin + at.row) * a.C + at.c;
        with_act(a.act, [&](auto act) { f.template write<decltype(act)::value>(a, v, 0, at.mine, y); });
    }
    cluster.barrier_wait();
}

// parts[n][rank][c] = (sum of dz, sum of dz xh) over the CTA's pixels, for norm_back_sum_parts; and dx.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 3) norm_back_resident(NormArgs a) {
    extern __shared__ uint4 smem4[];
    let_next_start();
    const int width = a.cols * V, lane = threadIdx.x % 32;
    // a thread's sums; the CTA's channels and groups: sums; the cluster's groups: p, q
    float2* s_sums = reinterpret_cast<float2*>(static_cast<Vec<T, V>*>(static_cast<void*>(smem4)) + 2 * a.held);
    float2 *s_chan = s_sums + a.quarter * V, *s_part = s_chan + width, *s_stat = s_part + a.groups;
    const Unit<V> at(a);
    Inputs<T, V> in(a, smem4, at.n, at.begin + at.row, at.c);
    float2 sb[kPairs<V>] = {}, sg[kPairs<V>] = {};
    if (at.mine) {
        const int half = (at.mine + 1) / 2;
        in.copy(a, 0, 0, half);
        copies_end();
        in.copy(a, 0, half, at.mine);
        copies_end();
        const Backward<V> f(a, at.n, at.c);
        with_act(a.act, [&](auto act) {
            as_they_come(at.mine, [&](int first, int end) { f.template sum_all<decltype(act)::value>(in.hx, in.hd, first, end, sb, sg); });
        });
    }
    put_sums<V>(a, at.row, at.col, s_sums, sb, sg);
    for (int j0 = threadIdx.x / 8; j0 < (width + 3) / 4 * 4; j0 += kThreads / 8) {            // eight lanes a channel
        const int j = min(j0, width - 1), col = j / V, i = j % V;
        const float2 s = sum_rows(a, s_sums, i, col);
        if (threadIdx.x % 8 == 0 && j0 < width) {
            s_chan[j] = s;
            const int c = at.slab * width + j;
            const float rstd = a.rstd[(int64_t)at.n * a.G + GroupOf(a, c).g];
            reinterpret_cast<float2*>(a.parts)[((int64_t)at.n * a.cluster + at.rank) * a.C + c] = make_float2(s.x, rstd * s.y);
        }
    }
    __syncthreads();
    for (int g = threadIdx.x / 32; g < a.groups; g += kWarps) {
        float2 s = {};
        for (int i = lane; i < a.cpg; i += 32)
            s = fma(both(a.gamma ? a.gamma[at.slab * width + g * a.cpg + i] : 1.0f), s_chan[g * a.cpg + i], s);
        s = sum_lanes<32>(s);
        if (lane == 0) s_part[g] = s;
    }
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    for (int g = threadIdx.x; g < a.groups; g += kThreads) {
        float2 s = {};
        for (int r = 0; r < a.cluster; ++r) s = add(s, *cluster.map_shared_rank(s_part + g, r));
        s_stat[g] = group_pq(a, s, a.rstd[(int64_t)at.n * a.G + at.slab * a.groups + g]);
    }
    __syncthreads();
    cluster.barrier_arrive();
    if (at.mine) {
        const Backward<V> f(a, at.n, at.c);
        const int first = at.slab * a.groups;
        float4 pq[kPairs<V>];
        pair_stats<V>(pq, a, at.c, [&](int g) { return s_stat[g - first]; });
        T* dx = static_cast<T*>(a.out) + ((int64_t)at.n * a.pixels + at.begin + at.row) * a.C + at.c;
        with_act(a.act, [&](auto act) { f.template write<decltype(act)::value>(a, in.hx, in.hd, 0, at.mine, dx, pq); });
    }
    cluster.barrier_wait();
}

__global__ void __launch_bounds__(kThreads) norm_back_sum_parts(NormArgs a) {
    wait_for_previous();
    norm_back_params(a, reinterpret_cast<const float2*>(a.parts), a.N * a.cluster, blockIdx.x);
}

// -------------------------------------------------------------------------------- launches

// Lets a kernel have all of an SM's shared memory; `done` remembers on which devices it may.
template <typename K>
cudaError_t allow_shared(K* kernel, std::atomic<uint64_t>& done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && !(dev < 64 && done.load() >> dev & 1)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormShared);
        if (e == cudaSuccess && dev < 64) done.fetch_or(uint64_t(1) << dev);
    }
    if (e != cudaSuccess) cudaGetLastError();
    return e;
}

// A kernel's launch: the first of a call, of CTAs in clusters, or one that starts before the end of the one before it.
constexpr int kFirst = 0, kNext = -1;
template <typename K, typename... Args>
cudaError_t launch_as(K* kernel, int how, dim3 grid, size_t smem, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    if (how == kNext) {
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
    } else {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)how;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    }
    cfg.attrs = attr;
    cfg.numAttrs = how > kFirst || (how == kNext && norm_starts_early()) ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...), l = cudaGetLastError();
    return e != cudaSuccess ? e : l;
}
template <typename K>
cudaError_t launch(K* kernel, std::atomic<uint64_t>& done, const NormArgs& a, int how, dim3 grid, size_t smem, cudaStream_t st) {
    if (const cudaError_t e = allow_shared(kernel, done)) return e;
    return launch_as(kernel, how, grid, smem, st, a);
}

template <typename T, int V, int NS>
cudaError_t forward(const NormArgs& a, cudaStream_t st) {
    static std::atomic<uint64_t> held{0}, sums{0}, result{0};
    const size_t smem = sizeof(Vec<T, V>) * a.held;
    if (a.cluster)
        return launch(norm_resident<T, V, NS>, held, a, a.cluster, dim3(a.cluster, a.slabs, a.N),
                      smem + (NS * kThreads + 2 * (size_t)a.groups + (size_t)a.cols * V) * sizeof(float2), st);
    const dim3 grid(a.chunks, a.tiles, a.N);
    if (const cudaError_t e = launch(norm_sums<T, V, NS>, sums, a, kFirst, grid, smem, st)) return e;
    if (const cudaError_t e = launch_as(norm_join, kNext, dim3(a.G, a.N), 0, st, a, V / NS)) return e;
    return launch(norm_result<T, V>, result, a, kNext, grid, smem, st);
}

template <typename T, int V>
cudaError_t backward(const NormArgs& a, cudaStream_t st) {
    static std::atomic<uint64_t> held{0}, sums{0}, result{0};
    const size_t smem = 2 * sizeof(Vec<T, V>) * a.held;
    if (a.cluster) {
        const cudaError_t e = launch(norm_back_resident<T, V>, held, a, a.cluster, dim3(a.cluster, a.slabs, a.N),
                                     smem + ((size_t)a.quarter * V + (size_t)a.cols * V + 2 * (size_t)a.groups) * sizeof(float2), st);
        if (e != cudaSuccess || !(a.dgamma || a.dbeta)) return e;
        return launch_as(norm_back_sum_parts, kNext, dim3((a.C + 31) / 32), 0, st, a);
    }
    const size_t beside = (size_t)a.quarter * V * sizeof(float2);
    if (const cudaError_t e = launch(norm_back_sums<T, V>, sums, a, kFirst, dim3(a.chunks, a.tiles, a.N), smem + beside, st)) return e;
    int bits = 0;
    while (1 << bits < a.cpg && 1 << bits < kThreads) ++bits;
    if (const cudaError_t e = launch_as(norm_back_join, kNext, dim3(a.G, a.N), 0, st, a, bits)) return e;
    return launch(norm_back_result<T, V>, result, a, kNext, dim3(a.chunks, a.tiles, a.N + 1), smem, st);
}

}  // namespace

template <typename T>
cudaError_t NormKernels<T>::forward(const NormArgs& a, int V, int NS, cudaStream_t st) {
    constexpr int W = 16 / sizeof(T);
    if (V == W) return NS == 1 ? patconv::forward<T, W, 1>(a, st) : patconv::forward<T, W, W>(a, st);
    if constexpr (sizeof(T) == 2)
        if (V == 2) return NS == 1 ? patconv::forward<T, 2, 1>(a, st) : patconv::forward<T, 2, 2>(a, st);
    return patconv::forward<T, 1, 1>(a, st);
}
template <typename T>
cudaError_t NormKernels<T>::backward(const NormArgs& a, int V, cudaStream_t st) {
    constexpr int W = 16 / sizeof(T);
    if (V == W) return patconv::backward<T, W>(a, st);
    if constexpr (sizeof(T) == 2)
        if (V == 2) return patconv::backward<T, 2>(a, st);
    return patconv::backward<T, 1>(a, st);
}

}  // namespace patconv
