// Kernels of norm.cu, for one type of activations each in norm_f32.cu, norm_f16.cu and norm_bf16.cu (three
// translation units, compiled side by side).
//
// The kernels are issue-bound before they are memory-bound if left to scalar code (27 instructions an
// element of a forward pass at 2.2 TB/s): the arithmetic runs on pairs of fp32 values, two to an
// instruction, the activation is chosen outside the loops, and exp and 1 / x are the hardware's
// approximations (2 and 1 ulp) with subnormals flushed.
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

namespace patconv {
namespace {

constexpr int kThreads = kNormThreads;
constexpr int kWarps = kThreads / 32;

// -------------------------------------------------------------------------------- vectors of values

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

// Asynchronous copies into the thread's own places of shared memory, which then extend its registers: no
// other thread reads them, so that waiting for the thread's own copies is all that is needed.
template <typename T, int V>
__device__ __forceinline__ void copy_async(Vec<T, V>* to, const T* from) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(to);
    if constexpr (sizeof(T) * V == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(from) : "memory");
    else if constexpr (sizeof(T) * V == 4)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(d), "l"(from) : "memory");
    else
        *to = load<T, V>(from);                                   // there is no copy of two bytes
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

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
        return mul(mul(dy, s), fma(z, add(both(1.0f), neg(s)), both(1.0f)));
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
    __device__ __forceinline__ Forward(const NormArgs& a, int c, Stat&& stat) {
        float m[2] = {}, s[2] = {}, b[2] = {};
        GroupOf at(a, c);
#pragma unroll
        for (int i = 0; i < V; ++i, at.next()) {
            const float2 st = stat(at.g);
            m[i % 2] = st.x;
            s[i % 2] = st.y * (a.gamma ? __ldg(a.gamma + c + i) : 1.0f);
            b[i % 2] = a.beta ? __ldg(a.beta + c + i) : 0.0f;
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
};

template <int V>
struct Backward {
    float2 mean[kPairs<V>], rstd[kPairs<V>], gamma[kPairs<V>], beta[kPairs<V>];
    __device__ __forceinline__ Backward(const NormArgs& a, int n, int c) {
        float m[2] = {}, r[2] = {}, g[2] = {}, b[2] = {};
        const float *mean_n = a.mean + (int64_t)n * a.G, *rstd_n = a.rstd + (int64_t)n * a.G;
        GroupOf at(a, c);
#pragma unroll
        for (int i = 0; i < V; ++i, at.next()) {
            m[i % 2] = -__ldg(mean_n + at.g);
            r[i % 2] = __ldg(rstd_n + at.g);
            g[i % 2] = a.gamma ? __ldg(a.gamma + c + i) : 1.0f;
            b[i % 2] = a.beta ? __ldg(a.beta + c + i) : 0.0f;
            mean[i / 2] = make_float2(m[0], m[1]);
            rstd[i / 2] = make_float2(r[0], r[1]);
            gamma[i / 2] = make_float2(g[0], g[1]);
            beta[i / 2] = make_float2(b[0], b[1]);
        }
    }
    // sums of dz and of dz xh
    template <int ACT, typename T>
    __device__ __forceinline__ void sum(const Vec<T, V>& x, const Vec<T, V>& dy, float2 (&sb)[kPairs<V>], float2 (&sg)[kPairs<V>]) const {
#pragma unroll
        for (int i = 0; i < kPairs<V>; ++i) {
            const float2 xh = mul(add(pair(x, i), mean[i]), rstd[i]);
            const float2 dz = through<ACT>(pair(dy, i), fma(xh, gamma[i], beta[i]));
            sb[i] = add(sb[i], dz);
            sg[i] = fma(dz, xh, sg[i]);
        }
    }
    // rstd (gamma dz - A / M - xh B / M); the product is rounded by itself, so that dx of a group of one value
    // is zero
    template <int ACT, typename T, typename Stat>
    __device__ __forceinline__ Vec<T, V> apply(Vec<T, V> x, const Vec<T, V>& dy, Stat&& stat) const {
#pragma unroll
        for (int i = 0; i < kPairs<V>; ++i) {
            const float2 xh = mul(add(pair(x, i), mean[i]), rstd[i]);
            const float2 dz = through<ACT>(pair(dy, i), fma(xh, gamma[i], beta[i]));
            const float4 ab = stat(i);                            // -A, -A', -B, -B'
            const float2 e = make_float2(__fmul_rn(gamma[i].x, dz.x), __fmul_rn(gamma[i].y, dz.y));
            const float2 d = fma(xh, make_float2(ab.z, ab.w), add(e, make_float2(ab.x, ab.y)));
            set_pair(x, i, mul(rstd[i], d));
        }
        return x;
    }
};
// A / M and B / M of a thread's groups, negative, by pairs of channels
template <int V, typename Stat>
__device__ __forceinline__ void pair_stats(float4 (&out)[kPairs<V>], const NormArgs& a, int c, Stat&& stat) {
    float A[2] = {}, B[2] = {};
    GroupOf at(a, c);
#pragma unroll
    for (int i = 0; i < V; ++i, at.next()) {
        const float2 s = stat(at.g);
        A[i % 2] = -s.x;
        B[i % 2] = -s.y;
        out[i / 2] = make_float4(A[0], A[1], B[0], B[1]);
    }
}
// [channel][thread] in shared memory: sums of dz, of dz xh
template <int V>
__device__ __forceinline__ void put_sums(float2* s, const float2 (&sb)[kPairs<V>], const float2 (&sg)[kPairs<V>]) {
#pragma unroll
    for (int i = 0; i < V; ++i)
        s[i * kThreads + threadIdx.x] = i % 2 ? make_float2(sb[i / 2].y, sg[i / 2].y) : make_float2(sb[i / 2].x, sg[i / 2].x);
}

// -------------------------------------------------------------------------------- streamed kernels

// One kernel for a whole call: its CTAs draw tickets, and the tickets' order is that of the work: the sums
// of `ahead` samples first, then by turns a sample's result and the sums of the next one, so that what is
// read for the sums is read again, for the result, while it is in L2.  The CTA that finishes a sample's
// last sum joins them.  A CTA that waits for a sample's sums holds a later ticket than all of those, so that
// they are done or at work, and the wait ends; should it not within a second, it is given up and recorded.
struct alignas(32) Item {
    int n, tile, chunk, kind;         // kSums, kResult, or kNone after the last
    int begin, base, rest, batches;   // pixels from begin on: base rows of each of the CTA's rows, one more of the
                                      // first `rest`; their batches
};
constexpr int kSums = 0, kResult = 1, kNone = 2;
__device__ __forceinline__ Item item_of(const NormArgs& a, uint32_t t, int batch) {
    const uint32_t per = (uint32_t)(a.chunks * a.tiles), first = per * a.ahead, pairs = (uint32_t)(a.N - a.ahead) * 2 * per;
    Item it;
    uint32_t r;
    if (t < first) {
        it.n = t / per;
        r = t - it.n * per;
        it.kind = kSums;
    } else if (t - first < pairs) {
        const uint32_t k = (t - first) / (2 * per);
        r = t - first - k * 2 * per;
        it.kind = r >= per ? kSums : kResult;
        it.n = r >= per ? k + a.ahead : k;
        if (r >= per) r -= per;
    } else {
        const uint32_t k = (t - first - pairs) / per;
        r = t - first - pairs - k * per;
        it.n = a.N - a.ahead + (int)k;
        it.kind = it.n >= a.N ? kNone : kResult;
    }
    it.chunk = a.tiles == 1 ? r : r / a.tiles;
    it.tile = a.tiles == 1 ? 0 : r % a.tiles;
    it.begin = it.chunk * a.chunk;
    const int count = (int)min((int64_t)a.chunk, a.pixels - it.begin);
    it.base = count / a.rows;
    it.rest = count - it.base * a.rows;
    it.batches = (it.base + (it.rest > 0) + batch - 1) / batch;
    return it;
}

constexpr long long kNormWaitCycles = 2000000000LL;              // about one second
__device__ __forceinline__ uint32_t load_acquire(const uint32_t* p) {
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void store_release(uint32_t* p, uint32_t v) {
    asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
// by one thread; false if the flag never came
__device__ __forceinline__ bool wait_flag(const uint32_t* flag, unsigned* status) {
    if (load_acquire(flag)) return true;
    const long long t0 = clock64();
    while (!load_acquire(flag)) {
        __nanosleep(64);
        if (clock64() - t0 > kNormWaitCycles) {
            atomicOr(status, kStatusNormTimeout);
            return false;
        }
    }
    return true;
}

struct Thread {                       // of a CTA: its column and its row
    int col, row;
    __device__ __forceinline__ explicit Thread(const NormArgs& a) {
        row = a.cols == 1 ? threadIdx.x : (int)__umulhi(threadIdx.x, a.cols_mul);
        col = threadIdx.x - row * a.cols;
    }
};
template <int V>
struct Place {                        // of a thread in an item: V channels from c, `mine` pixels from its row on
    int c, mine;
    __device__ __forceinline__ Place(const NormArgs& a, const Thread& th, const Item& it) {
        c = (it.tile * a.cols + th.col) * V;
        mine = th.row < a.rows && c < a.C ? it.base + (th.row < it.rest) : 0;
    }
    Place() = default;
};

// Keeps copies of kDepth - 1 batches of U vectors a thread of each input under way, across the items'
// borders: the load side (an item and a batch) runs ahead of the side that computes.  One thread draws
// tickets, `draw` items ahead, as many as the load side can get ahead and one; a ticket is read after the
// barrier that follows its writing (every item has one).
constexpr int kDepth = kStreamDepth, kTickets = 8;
static_assert(kDepth < kTickets, "tickets are drawn at most kDepth items ahead");

template <typename T, int V, int U, int INPUTS>
struct Pipe {
    const NormArgs& a;
    const Thread th;
    Vec<T, V>* mine;                  // the thread's places: [kDepth][INPUTS][U][kThreads]
    Item* items;                      // shared, kTickets of them
    uint32_t drawn = 0;               // one thread: a ticket under way
    int ahead_item = 0, ahead_batch = 0, ahead_batches, ahead_left, ahead_slot = 0, slot = 0;
    const T *x, *dy;                  // of the load side: its next vectors
    const int64_t x_step, dy_step;

    __device__ __forceinline__ Pipe(const NormArgs& args, void* smem, Item* s_items)
        : a(args), th(args), mine(static_cast<Vec<T, V>*>(smem) + threadIdx.x), items(s_items),
          x_step(args.rows * args.x_pixel), dy_step(args.rows * args.dy_pixel) {
        if (threadIdx.x == 0) {
            const uint32_t t = atomicAdd(a.counters, a.draw);
            for (int i = 0; i < a.draw; ++i) items[i] = item_of(a, t + i, U);
            drawn = atomicAdd(a.counters, 1);
        }
        __syncthreads();
        enter();
        for (int i = 0; i < kDepth - 1; ++i) advance();
    }
    __device__ __forceinline__ void enter() {
        const Item it = items[ahead_item % kTickets];
        const Place<V> at(a, th, it);
        ahead_batch = 0;
        ahead_batches = it.kind == kNone ? -1 : it.batches;       // after a last ticket come last ones
        ahead_left = it.kind == kNone ? 0 : at.mine;
        const int64_t p = it.begin + th.row;
        x = static_cast<const T*>(a.x) + it.n * a.x_sample + p * a.x_pixel + at.c;
        if constexpr (INPUTS == 2) dy = static_cast<const T*>(a.dy) + it.n * a.dy_sample + p * a.dy_pixel + at.c;
    }
    // the next batch's copies
    __device__ __forceinline__ void advance() {
        if (ahead_batch == ahead_batches) {
            ++ahead_item;
            enter();
        }
        Vec<T, V>* to = mine + ahead_slot * (INPUTS * U * kThreads);
        const auto copy = [&](auto k) {
#pragma unroll
            for (int u = 0; u < U; ++u, x += x_step)
                if (u < k) copy_async(to + u * kThreads, x);
            if constexpr (INPUTS == 2) {
#pragma unroll
                for (int u = 0; u < U; ++u, dy += dy_step)
                    if (u < k) copy_async(to + (U + u) * kThreads, dy);
            }
        };
        if (ahead_left >= U)
            copy(std::integral_constant<int, U>());
        else if (ahead_left > 0)
            copy(ahead_left);
        copies_end();
        ahead_left -= U;
        ++ahead_batch;
        ahead_slot = ahead_slot + 1 == kDepth ? 0 : ahead_slot + 1;
    }
    // the item that is next to compute; `i` counts them
    __device__ __forceinline__ Item begin(int i) {
        if (threadIdx.x == 0) {
            items[(i + a.draw) % kTickets] = item_of(a, drawn, U);
            drawn = atomicAdd(a.counters, 1);
        }
        return items[i % kTickets];
    }
    // the item's batches: f(first vector, vectors), a constant U but for the last
    template <typename F>
    __device__ __forceinline__ void each(const Item& it, int left, F&& f) {
#pragma unroll 1
        for (int b = 0; b < it.batches; ++b, left -= U) {
            advance();
            copies_wait<kDepth - 1>();
            if (left >= U)
                f(b * U, std::integral_constant<int, U>());
            else if (left > 0)
                f(b * U, left);
            slot = slot + 1 == kDepth ? 0 : slot + 1;
        }
    }
    __device__ __forceinline__ Vec<T, V> get(int input, int u) const {
        return mine[((slot * INPUTS + input) * U + u) * kThreads];
    }
    static constexpr size_t kBytes = sizeof(Vec<T, V>) * kDepth * INPUTS * U * kThreads;
};

// Whether this CTA has finished the last of `per` parts of a sample: then it sees all of them.  The barrier
// puts the CTA's writes before the one thread's fence; a fence of every thread would wait for its copies.
__device__ __forceinline__ bool last_of(uint32_t* done, uint32_t per) {
    __syncthreads();
    bool last = false;
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(done, 1) == per - 1;
        __threadfence();
    }
    return __syncthreads_or(last);
}

template <typename T, int V, int NS>
__global__ void __launch_bounds__(kThreads, 2) norm_stream(NormArgs a) {
    constexpr int S = V / NS, U = kStreamBatch;
    extern __shared__ uint4 smem4[];
    __shared__ float2 s_sets[NS * kThreads];
    __shared__ int s_mine[kThreads];
    __shared__ Item s_items[kTickets];
    Pipe<T, V, U, 1> pipe(a, smem4, s_items);
    uint32_t *done = a.counters + 2, *ready = done + a.N;
    const int sets = a.C / S;                                     // of a row
    for (int i = 0;; ++i) {
        const Item it = pipe.begin(i);
        if (it.kind == kNone) break;
        const Place<V> at(a, pipe.th, it);
        if (it.kind == kSums) {
            Sets<T, V, NS> m;
            pipe.each(it, at.mine, [&](int, auto k) {
                Vec<T, V> v[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u < k) v[u] = pipe.get(0, u);
                m.take(v, k);
            });
            m.put(s_sets);
            s_mine[threadIdx.x] = at.mine * S;
            __syncthreads();
            // eight lanes a set, over the rows
            const int here = min(a.cols, a.C / V - it.tile * a.cols) * NS;
            for (int j0 = threadIdx.x / 8; j0 < (here + 3) / 4 * 4; j0 += kThreads / 8) {
                const int j = min(j0, here - 1), col = j / NS, k = j % NS;
                Moments m{0.0f, 0.0f, 0.0f};
                for (int r = threadIdx.x % 8; r < a.rows; r += 8) {
                    const int t = r * a.cols + col;
                    const float2 s = s_sets[k * kThreads + t];
                    m = join(m, {(float)s_mine[t], s.x, s.y});
                }
                m = join_lanes<8>(m);
                if (threadIdx.x % 8 == 0 && j0 < here)
                    reinterpret_cast<float2*>(a.parts)[((int64_t)it.n * a.chunks + it.chunk) * sets + it.tile * a.cols * NS + j] =
                        make_float2(m.mean, m.m2);
            }
            if (!last_of(done + it.n, a.chunks * a.tiles)) continue;
            const float2* parts = reinterpret_cast<const float2*>(a.parts) + (int64_t)it.n * a.chunks * sets;
            // eight lanes a group, over its sets where they are many, else over the stretches
            const int lane = threadIdx.x % 8;
            const bool wide = a.spg >= 8;
            for (int g0 = threadIdx.x / 8; g0 < (a.G + 3) / 4 * 4; g0 += kThreads / 8) {
                const int g = min(g0, a.G - 1);
                Moments m{0.0f, 0.0f, 0.0f};
                for (int o = 0; o < (wide ? a.chunks : a.spg); ++o) {
                    const int count = wide ? a.spg : a.chunks;
#pragma unroll 8
                    for (int e = lane; e < count; e += 8) {
                        const int k = wide ? o : e, set = g * a.spg + (wide ? e : o);
                        const float2 p = __ldcg(parts + (int64_t)k * sets + set);
                        const int64_t left = a.pixels - (int64_t)k * a.chunk;
                        m = join(m, {(float)(left < a.chunk ? left : a.chunk) * S, p.x, p.y});
                    }
                }
                m = join_lanes<8>(m);
                if (lane == 0 && g0 < a.G) {
                    const float var = m.m2 / ((float)a.pixels * a.cpg);
                    a.mean_out[(int64_t)it.n * a.G + g] = m.mean;
                    a.rstd_out[(int64_t)it.n * a.G + g] = 1.0f / sqrtf(var + a.eps);
                }
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                __threadfence();
                store_release(ready + it.n, 1);
            }
        } else {
            const bool good = __syncthreads_and(threadIdx.x != 0 || wait_flag(ready + it.n, a.status));
            const float *mean = a.mean_out + (int64_t)it.n * a.G, *rstd = a.rstd_out + (int64_t)it.n * a.G;
            const int c = min(at.c, a.C - V);                     // of a thread without a column: any
            const Forward<V> f(a, c, [&](int g) { return make_float2(__ldcg(mean + g), __ldcg(rstd + g)); });
            T* y = static_cast<T*>(a.out) + ((int64_t)it.n * a.pixels + it.begin + pipe.th.row) * a.C + at.c;
            const int64_t y_step = (int64_t)a.rows * a.C;
            with_act(a.act, [&](auto act) {
                pipe.each(it, at.mine, [&](int first, auto k) {
                    T* to = y + first * y_step;
#pragma unroll
                    for (int u = 0; u < U; ++u, to += y_step)
                        if (u < k && good) store<T, V>(to, f.template apply<decltype(act)::value>(pipe.get(0, u)));
                });
            });
        }
    }
    copies_wait<0>();
}

// sums: [N][C] (dz, dz xh), then [N][G] (A / M, B / M)
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 2) norm_back_stream(NormArgs a) {
    constexpr int U = kStreamBatch / 2;
    extern __shared__ uint4 smem4[];
    __shared__ float2 s_sums[V * kThreads];
    __shared__ Item s_items[kTickets];
    Pipe<T, V, U, 2> pipe(a, smem4, s_items);
    uint32_t *joined = a.counters + 1, *done = a.counters + 2, *ready = done + a.N;
    float2 *channel = reinterpret_cast<float2*>(a.sums), *group = channel + (int64_t)a.N * a.C;
    for (int i = 0;; ++i) {
        const Item it = pipe.begin(i);
        if (it.kind == kNone) break;
        const Place<V> at(a, pipe.th, it);
        const int own_c = min(at.c, a.C - V);                     // of a thread without a column: any
        if (it.kind == kSums) {
            float2 sb[kPairs<V>] = {}, sg[kPairs<V>] = {};
            const Backward<V> f(a, it.n, own_c);
            with_act(a.act, [&](auto act) {
                pipe.each(it, at.mine, [&](int, auto k) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (u < k) f.template sum<decltype(act)::value>(pipe.get(0, u), pipe.get(1, u), sb, sg);
                });
            });
            put_sums<V>(s_sums, sb, sg);
            __syncthreads();
            const int here = min(a.cols * V, a.C - it.tile * a.cols * V);
            for (int j0 = threadIdx.x / 8; j0 < (here + 3) / 4 * 4; j0 += kThreads / 8) {
                const int j = min(j0, here - 1), col = j / V, i = j % V;
                float2 s = {};
                for (int r = threadIdx.x % 8; r < a.rows; r += 8) s = add(s, s_sums[i * kThreads + r * a.cols + col]);
                s = sum_lanes<8>(s);
                if (threadIdx.x % 8 == 0 && j0 < here)
                    reinterpret_cast<float2*>(a.parts)[((int64_t)it.n * a.chunks + it.chunk) * a.C + it.tile * a.cols * V + j] = s;
            }
            if (!last_of(done + it.n, a.chunks * a.tiles)) continue;
            // the sample's channels, eight lanes a channel over the stretches, then its groups
            const float2* parts = reinterpret_cast<const float2*>(a.parts) + (int64_t)it.n * a.chunks * a.C;
            for (int c0 = threadIdx.x / 8; c0 < (a.C + 3) / 4 * 4; c0 += kThreads / 8) {
                const int c = min(c0, a.C - 1);
                float2 s = {};
#pragma unroll 8
                for (int k = threadIdx.x % 8; k < a.chunks; k += 8) s = add(s, __ldcg(parts + (int64_t)k * a.C + c));
                s = sum_lanes<8>(s);
                if (threadIdx.x % 8 == 0 && c0 < a.C) channel[(int64_t)it.n * a.C + c] = s;
            }
            __syncthreads();
            for (int g = threadIdx.x / 32; g < a.G; g += kWarps) {
                float2 s = {};
                for (int i = threadIdx.x % 32; i < a.cpg; i += 32) {
                    const int c = g * a.cpg + i;
                    s = fma(both(a.gamma ? a.gamma[c] : 1.0f), channel[(int64_t)it.n * a.C + c], s);
                }
                s = sum_lanes<32>(s);
                if (threadIdx.x % 32 == 0) group[(int64_t)it.n * a.G + g] = mul(s, both(1.0f / ((float)a.pixels * a.cpg)));
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                __threadfence();
                store_release(ready + it.n, 1);
            }
            if (!(a.dgamma || a.dbeta) || !last_of(joined, a.N)) continue;
            for (int c0 = threadIdx.x / 8; c0 < (a.C + 3) / 4 * 4; c0 += kThreads / 8) {      // over the samples
                const int c = min(c0, a.C - 1);
                float2 s = {};
#pragma unroll 4
                for (int n = threadIdx.x % 8; n < a.N; n += 8) s = add(s, __ldcg(channel + (int64_t)n * a.C + c));
                s = sum_lanes<8>(s);
                if (threadIdx.x % 8 || c0 >= a.C) continue;
                if (a.dbeta) a.dbeta[c] = s.x;
                if (a.dgamma) a.dgamma[c] = s.y;
            }
        } else {
            const bool good = __syncthreads_and(threadIdx.x != 0 || wait_flag(ready + it.n, a.status));
            const Backward<V> f(a, it.n, own_c);
            float4 ab[kPairs<V>];
            pair_stats<V>(ab, a, own_c, [&](int g) { return __ldcg(group + (int64_t)it.n * a.G + g); });
            T* dx = static_cast<T*>(a.out) + ((int64_t)it.n * a.pixels + it.begin + pipe.th.row) * a.C + at.c;
            const int64_t dx_step = (int64_t)a.rows * a.C;
            with_act(a.act, [&](auto act) {
                pipe.each(it, at.mine, [&](int first, auto k) {
                    T* to = dx + first * dx_step;
#pragma unroll
                    for (int u = 0; u < U; ++u, to += dx_step)
                        if (u < k && good)
                            store<T, V>(to, f.template apply<decltype(act)::value>(pipe.get(0, u), pipe.get(1, u),
                                                                                 [&](int i) { return ab[i]; }));
                });
            });
        }
    }
    copies_wait<0>();
}

// -------------------------------------------------------------------------------- resident kernels

namespace cg = cooperative_groups;

// A unit of the resident kernels is a sample's slab: `cols` vectors of every pixel, whole groups.  The CTAs
// of a cluster take a stretch of its pixels each and hold it in registers between the sums and the
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

template <typename T, int V, int NS, int K>
__global__ void __launch_bounds__(kThreads, K * V * sizeof(T) > 128 ? 2 : 3) norm_resident(NormArgs a) {
    constexpr int S = V / NS;
    extern __shared__ float2 smem2[];
    float2 *s_sets = smem2, *s_part = s_sets + NS * kThreads;     // a thread's sets; the CTA's groups: mean, m2
    float2* s_stat = s_part + a.groups;                           // the cluster's groups: mean, rstd
    __shared__ int s_mine[kThreads];
    const Unit<V> at(a);
    const int lane = threadIdx.x % 32;
    const T* x = static_cast<const T*>(a.x) + at.n * a.x_sample + (at.begin + at.row) * a.x_pixel + at.c;
    const int64_t step = a.rows * a.x_pixel;
    Vec<T, V> v[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k < at.mine) v[k] = load<T, V>(x + k * step);
    {
        Sets<T, V, NS> m;
        m.take(v, at.mine);
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
        const Forward<V> f(a, at.c, [&](int g) { return s_stat[g - first]; });
        T* y = static_cast<T*>(a.out) + ((int64_t)at.n * a.pixels + at.begin + at.row) * a.C + at.c;
        const int64_t y_step = (int64_t)a.rows * a.C;
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (k < at.mine) store<T, V>(y + k * y_step, f.template apply<decltype(act)::value>(v[k]));
        });
    }
    cluster.barrier_wait();
}

// parts[n][rank][c] = (sum of dz, sum of dz xh) over the CTA's pixels, for norm_back_params; and dx.
template <typename T, int V, int K>
__global__ void __launch_bounds__(kThreads, 2) norm_back_resident(NormArgs a) {
    extern __shared__ float2 smem2[];
    const int width = a.cols * V, lane = threadIdx.x % 32;
    float2 *s_sums = smem2, *s_chan = s_sums + V * kThreads;      // a thread's sums; the CTA's channels
    float2 *s_part = s_chan + width, *s_stat = s_part + a.groups; // the CTA's groups: A, B; the cluster's
    const Unit<V> at(a);
    const T* x = static_cast<const T*>(a.x) + at.n * a.x_sample + (at.begin + at.row) * a.x_pixel + at.c;
    const T* dy = static_cast<const T*>(a.dy) + at.n * a.dy_sample + (at.begin + at.row) * a.dy_pixel + at.c;
    const int64_t x_step = a.rows * a.x_pixel, dy_step = a.rows * a.dy_pixel;
    Vec<T, V> v[K], w[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k < at.mine) {
            v[k] = load<T, V>(x + k * x_step);
            w[k] = load<T, V>(dy + k * dy_step);
        }
    float2 sb[kPairs<V>] = {}, sg[kPairs<V>] = {};
    if (at.mine) {
        const Backward<V> f(a, at.n, at.c);
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (k < at.mine) f.template sum<decltype(act)::value>(v[k], w[k], sb, sg);
        });
    }
    put_sums<V>(s_sums, sb, sg);
    __syncthreads();
    for (int j0 = threadIdx.x / 8; j0 < (width + 3) / 4 * 4; j0 += kThreads / 8) {            // eight lanes a channel
        const int j = min(j0, width - 1), col = j / V, i = j % V;
        float2 s = {};
        for (int r = threadIdx.x % 8; r < a.rows; r += 8) s = add(s, s_sums[i * kThreads + r * a.cols + col]);
        s = sum_lanes<8>(s);
        if (threadIdx.x % 8 == 0 && j0 < width) {
            s_chan[j] = s;
            reinterpret_cast<float2*>(a.parts)[((int64_t)at.n * a.cluster + at.rank) * a.C + at.slab * width + j] = s;
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
    const float2 inv = both(1.0f / ((float)a.pixels * a.cpg));
    for (int g = threadIdx.x; g < a.groups; g += kThreads) {
        float2 s = {};
        for (int r = 0; r < a.cluster; ++r) s = add(s, *cluster.map_shared_rank(s_part + g, r));
        s_stat[g] = mul(s, inv);
    }
    __syncthreads();
    cluster.barrier_arrive();
    if (at.mine) {
        const Backward<V> f(a, at.n, at.c);
        const int first = at.slab * a.groups;
        float4 ab[kPairs<V>];
        pair_stats<V>(ab, a, at.c, [&](int g) { return s_stat[g - first]; });
        T* dx = static_cast<T*>(a.out) + ((int64_t)at.n * a.pixels + at.begin + at.row) * a.C + at.c;
        const int64_t dx_step = (int64_t)a.rows * a.C;
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (k < at.mine)
                    store<T, V>(dx + k * dx_step, f.template apply<decltype(act)::value>(v[k], w[k], [&](int i) { return ab[i]; }));
        });
    }
    cluster.barrier_wait();
}

// dgamma and dbeta from the parts of norm_back_resident, in their order: a warp takes 32 channels, the
// CTA's warps the parts in turn.
__global__ void __launch_bounds__(kThreads) norm_back_params(NormArgs a) {
    __shared__ float2 s[kThreads];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, parts = a.N * a.cluster;
    float2 sum = {};
    if (c < a.C)
        for (int k = threadIdx.x / 32; k < parts; k += kWarps)
            sum = add(sum, reinterpret_cast<const float2*>(a.parts)[(int64_t)k * a.C + c]);
    s[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x >= 32 || c >= a.C) return;
    for (int w = 1; w < kWarps; ++w) sum = add(sum, s[w * 32 + threadIdx.x]);
    if (a.dbeta) a.dbeta[c] = sum.x;
    if (a.dgamma) a.dgamma[c] = sum.y;
}

// -------------------------------------------------------------------------------- launches

// Lets a kernel have `bytes` of dynamic shared memory on the current device; `allowed` remembers the devices.
template <typename K>
cudaError_t allow_shared(K* kernel, size_t bytes, std::atomic<uint64_t>& allowed) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && !(dev < 64 && allowed.load() >> dev & 1)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e == cudaSuccess && dev < 64) allowed.fetch_or(uint64_t(1) << dev);
    }
    if (e != cudaSuccess) cudaGetLastError();
    return e;
}

template <typename... A>
cudaError_t launch_clusters(void (*kernel)(A...), const NormArgs& a, size_t smem, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.cluster, (unsigned)a.slabs, (unsigned)a.N);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a), l = cudaGetLastError();
    return e != cudaSuccess ? e : l;
}

template <typename T, int V, int NS>
cudaError_t forward_held(const NormArgs& a, int K, cudaStream_t st) {
    const size_t smem = (NS * kThreads + 2 * (size_t)a.groups) * sizeof(float2);
    if constexpr (V * sizeof(T) == 16) {
        switch (K) {
            case 2: return launch_clusters(norm_resident<T, V, NS, 2>, a, smem, st);
            case 4: return launch_clusters(norm_resident<T, V, NS, 4>, a, smem, st);
            case 8: return launch_clusters(norm_resident<T, V, NS, 8>, a, smem, st);
            case 16: return launch_clusters(norm_resident<T, V, NS, 16>, a, smem, st);
        }
    } else {
        switch (K) {
            case 8: return launch_clusters(norm_resident<T, V, NS, 8>, a, smem, st);
            case 32: return launch_clusters(norm_resident<T, V, NS, 32>, a, smem, st);
        }
    }
    return cudaErrorInvalidValue;
}

template <typename T, int V>
cudaError_t backward_held(const NormArgs& a, int K, cudaStream_t st) {
    const size_t smem = (V * kThreads + (size_t)a.cols * V + 2 * (size_t)a.groups) * sizeof(float2);
    cudaError_t e = cudaErrorInvalidValue;
    if constexpr (V * sizeof(T) == 16) {
        switch (K) {
            case 2: e = launch_clusters(norm_back_resident<T, V, 2>, a, smem, st); break;
            case 4: e = launch_clusters(norm_back_resident<T, V, 4>, a, smem, st); break;
            case 8: e = launch_clusters(norm_back_resident<T, V, 8>, a, smem, st); break;
        }
    } else {
        switch (K) {
            case 8: e = launch_clusters(norm_back_resident<T, V, 8>, a, smem, st); break;
            case 24: e = launch_clusters(norm_back_resident<T, V, 24>, a, smem, st); break;
        }
    }
    if (e != cudaSuccess || !(a.dgamma || a.dbeta)) return e;
    norm_back_params<<<(a.C + 31) / 32, kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t zero_counters(const NormArgs& a, cudaStream_t st) {
    const cudaError_t e = cudaMemsetAsync(a.counters, 0, norm_counters(a.N) * sizeof(uint32_t), st);
    if (e != cudaSuccess) cudaGetLastError();
    return e;
}
template <typename T, int V, int NS>
cudaError_t forward_streamed(const NormArgs& a, cudaStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    constexpr size_t smem = Pipe<T, V, kStreamBatch, 1>::kBytes;
    if (const cudaError_t e = allow_shared(norm_stream<T, V, NS>, smem, allowed)) return e;
    if (const cudaError_t e = zero_counters(a, st)) return e;
    norm_stream<T, V, NS><<<a.grid, kThreads, smem, st>>>(a);
    return cudaGetLastError();
}
template <typename T, int V>
cudaError_t backward_streamed(const NormArgs& a, cudaStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    constexpr size_t smem = Pipe<T, V, kStreamBatch / 2, 2>::kBytes;
    if (const cudaError_t e = allow_shared(norm_back_stream<T, V>, smem, allowed)) return e;
    if (const cudaError_t e = zero_counters(a, st)) return e;
    norm_back_stream<T, V><<<a.grid, kThreads, smem, st>>>(a);
    return cudaGetLastError();
}

}  // namespace

template <typename T>
cudaError_t NormKernels<T>::forward(const NormArgs& a, int V, int NS, int K, cudaStream_t st) {
    constexpr int W = 16 / sizeof(T);
    if (V == W) {
        if (K) return NS == 1 ? forward_held<T, W, 1>(a, K, st) : forward_held<T, W, W>(a, K, st);
        return NS == 1 ? forward_streamed<T, W, 1>(a, st) : forward_streamed<T, W, W>(a, st);
    }
    if constexpr (sizeof(T) == 2)
        if (V == 2) {
            if (K) return NS == 1 ? forward_held<T, 2, 1>(a, K, st) : forward_held<T, 2, 2>(a, K, st);
            return NS == 1 ? forward_streamed<T, 2, 1>(a, st) : forward_streamed<T, 2, 2>(a, st);
        }
    return K ? forward_held<T, 1, 1>(a, K, st) : forward_streamed<T, 1, 1>(a, st);
}
template <typename T>
cudaError_t NormKernels<T>::backward(const NormArgs& a, int V, int K, cudaStream_t st) {
    constexpr int W = 16 / sizeof(T);
    if (V == W) return K ? backward_held<T, W>(a, K, st) : backward_streamed<T, W>(a, st);
    if constexpr (sizeof(T) == 2)
        if (V == 2) return K ? backward_held<T, 2>(a, K, st) : backward_streamed<T, 2>(a, st);
    return K ? backward_held<T, 1>(a, K, st) : backward_streamed<T, 1>(a, st);
}

}  // namespace patconv
