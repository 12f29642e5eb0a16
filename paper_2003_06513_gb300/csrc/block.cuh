// Kernels of block.cu, for one type of blocks and stream each in block_f32.cu, block_f16.cu, block_f16_f32.cu and so on: five
// translation units, compiled side by side.
//
// A row -- a pixel's channels -- is taken by `threads` threads of eight channels each: a power of two of them inside a
// warp for rows of up to 256 channels, whole warps for longer ones.  All of a row is in registers between its readings
// and the results, the four sums that two norms and their gradients take go over the lanes by shuffles and, in longer
// rows, over the warps through shared memory.
#pragma once

#include <algorithm>
#include <atomic>

#include "block.h"
#include "patconv.h"
#include "vec.cuh"

namespace patconv {
namespace {

constexpr int E = kBlockEight;

// Forms of the kernels.  kLong: a CTA has one row, of whole warps.  kShort: several rows, of a power of two of threads each.
// 1 to 32: the same with so many threads, known beforehand.  KIND kStrided: any strides; kDense: one offset for all tensors; kRms and
// kLayer: dense, both norms of this kind and all inputs there.  With loops that unroll, one 32-bit offset for all tensors and no
// choices left a row takes half the instructions, and its chain of dependent ones, which bounds the kernels, is shorter (32 x 256 x
// 56 x 56 forward: 58 us to 44 with known forms and the parameters in shared memory).
enum { kLong = -1, kShort = 0 };
enum { kStrided = 0, kRms = PP_NORM_RMS, kLayer = PP_NORM_LAYER, kDense = 3 };

// eight channels of a row: V adjacent ones, then those `threads` vectors on, and so on
struct Eight {
    float2 v[E / 2];
};
template <int V>
__device__ __forceinline__ int channel(int lane, int threads, int k) {
    return (lane + k / V * threads) * V + k % V;
}
template <typename T, int V>
struct Raw {                                          // as it is read
    Vec<T, V> v[E / V];
};
// What a thread reads of an input, a round ahead of its use: asynchronous copies of 4 to 16 bytes into the thread's own
// places of shared memory, which no other thread reads, so that waiting for its own copies is all that is needed, and what
// is under way costs no registers.  There is no copy of two bytes: single halves are read when they are used.
template <typename T, int V>
struct Ahead {
    static_assert(sizeof(T) * V <= 16);
    static constexpr int S = sizeof(T) * V, P = E / V;
    static constexpr bool kAsync = S >= 4;
    static constexpr int kBytes = kAsync ? E * (int)sizeof(T) : 0;       // of a thread and round
    // channels from the thread's first one to piece k
    static __device__ __forceinline__ int apart(int threads, int k) { return k * threads * V; }
    // the thread's own channels from `mine` on, those that `live(k)` says are there; what is not copied becomes 0
    template <typename Live>
    static __device__ __forceinline__ void ask(uint32_t place, const T* mine, int threads, Live&& live) {
        if constexpr (kAsync) {
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const bool wanted = live(k);
                const T* from = wanted ? mine + apart(threads, k) : mine;
                const uint32_t to = place + (k * blockDim.x + threadIdx.x) * S;
                const int n = wanted ? S : 0;
                if constexpr (S == 16)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n) : "memory");
                else
                    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(S), "r"(n) : "memory");
            }
        }
    }
    // the k-th of the thread's eight values
    static __device__ __forceinline__ float one(uint32_t place, const T* mine, int threads, int k) {
        if constexpr (!kAsync) {
            return widen(mine[apart(threads, k)]);
        } else {
            const int byte = k * (int)sizeof(T), from = place + ((byte / S) * blockDim.x + threadIdx.x) * S + byte % S;
            if constexpr (sizeof(T) == 4) {
                float x;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(from) : "memory");
                return x;
            } else {
                uint16_t bits;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(bits) : "r"(from) : "memory");
                T x;
                memcpy(&x, &bits, 2);
                return widen(x);
            }
        }
    }
    template <typename Live>
    static __device__ __forceinline__ Raw<T, V> get(uint32_t place, const T* mine, int threads, Live&& live) {
        Raw<T, V> r;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            char* to = reinterpret_cast<char*>(&r) + k * S;
            const uint32_t from = place + (k * blockDim.x + threadIdx.x) * S;
            if constexpr (S == 16) {
                uint4 v;
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from) : "memory");
                memcpy(to, &v, 16);
            } else if constexpr (S == 8) {
                uint2 v;
                asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(from) : "memory");
                memcpy(to, &v, 8);
            } else if constexpr (S == 4) {
                uint32_t v;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(from) : "memory");
                memcpy(to, &v, 4);
            } else {
                T v = T(0.0f);
                if (live(k)) v = mine[apart(threads, k)];
                memcpy(to, &v, S);
            }
        }
        return r;
    }
};
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// Rounds of rows that a CTA has in its ring: four, and in the backward pass, with four tensors and not two, three; two there where
// 512 threads with all of it in fp32 would take more shared memory than an SM has.
constexpr int kRounds = 4;
template <typename TX, typename TB, bool WIDE>
constexpr int kRoundsBack = WIDE && sizeof(TX) + sizeof(TB) == 8 ? 2 : 3;

template <typename T, int V>
__device__ __forceinline__ Eight widened(const Raw<T, V>& r) {
    Eight e;
    if constexpr (V == 1) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) e.v[i] = make_float2(widen(r.v[2 * i].v[0]), widen(r.v[2 * i + 1].v[0]));
    } else {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) e.v[i] = pair(r.v[2 * i / V], 2 * i % V / 2);
    }
    return e;
}
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> narrowed(const Eight& e) {
    Raw<T, V> r;
    if constexpr (V == 1) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            narrow(e.v[i].x, r.v[2 * i].v[0]);
            narrow(e.v[i].y, r.v[2 * i + 1].v[0]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) set_pair(r.v[2 * i / V], 2 * i % V / 2, e.v[i]);
    }
    return r;
}
template <typename T, int V, typename Live>
__device__ __forceinline__ void put(T* mine, const Raw<T, V>& r, int threads, Live&& live) {
#pragma unroll
    for (int j = 0; j < E / V; ++j) {
        if (!live(j)) continue;
        store<T, V>(mine + j * threads * V, r.v[j]);
    }
}
// a parameter's values, `otherwise` where there is none, and beyond the row 0
template <int V>
__device__ __forceinline__ Eight parameter(const float* p, float otherwise, int lane, const BlockArgs& a) {
    Eight e;
    float* f = reinterpret_cast<float*>(e.v);
#pragma unroll
    for (int k = 0; k < E; ++k) {
        const int c = channel<V>(lane, a.threads, k);
        f[k] = c < a.C ? (p ? p[c] : otherwise) : 0.0f;
    }
    return e;
}
// A parameter's values where they are used: of a long row in the thread's registers, of short ones in shared memory, where the
// CTA's rows share them: three parameters fewer, 24 registers of the 128 that a thread has.
template <int FORM>
struct Held {
    Eight e;
    uint32_t place;                                   // this thread's first four values, the others `threads` places on
    __device__ __forceinline__ Held(float* shared, int lane) : place((uint32_t)__cvta_generic_to_shared(shared) + lane * 16) {}
    // by every thread of a long row, by those of one of the short ones; a barrier before they are used
    __device__ __forceinline__ void set(const Eight& v, int threads, bool mine) {
        if (FORM == kLong) {
            e = v;
        } else if (mine) {
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(place), "f"(v.v[0].x), "f"(v.v[0].y), "f"(v.v[1].x), "f"(v.v[1].y) : "memory");
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(place + threads * 16), "f"(v.v[2].x), "f"(v.v[2].y), "f"(v.v[3].x), "f"(v.v[3].y) : "memory");
        }
    }
    __device__ __forceinline__ Eight get(int threads) const {
        if (FORM == kLong) return e;
        Eight v;
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.v[0].x), "=f"(v.v[0].y), "=f"(v.v[1].x), "=f"(v.v[1].y) : "r"(place) : "memory");
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.v[2].x), "=f"(v.v[2].y), "=f"(v.v[3].x), "=f"(v.v[3].y) : "r"(place + threads * 16) : "memory");
        return v;
    }
};
template <int FORM>
constexpr int kHeldFloats = FORM == kLong ? 1 : FORM == kShort ? 32 * E : FORM * E;
template <int V>
__device__ __forceinline__ Eight times(const Eight& p, const Eight& q) {
    Eight r;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) r.v[i] = mul(p.v[i], q.v[i]);
    return r;
}
// whether each of the eight is one of the row's channels
template <int V>
__device__ __forceinline__ bool inside(int lane, const BlockArgs& a, int k) { return lane + k / V * a.threads < a.vectors; }

template <int V>
__device__ __forceinline__ float own_channels(int lane, const BlockArgs& a) {
    int n = 0;
    for (int k = 0; k < E; ++k) n += inside<V>(lane, a, k);
    return (float)n;
}

// Sums over a row's threads, to all of them, in a fixed order.
template <int FORM>
struct RowSum {
    static constexpr bool WIDE = FORM == kLong;
    int threads;
    float* scratch;                                   // kLong: 2 x 64
    int turn = 0;
    template <typename T, int K>
    __device__ __forceinline__ void over_lanes(T (&s)[K]) const {
        if constexpr (FORM == kShort) {
            for (int o = 1; o < threads; o *= 2)
#pragma unroll
                for (int k = 0; k < K; ++k) s[k] += __shfl_xor_sync(0xffffffffu, s[k], o);
        } else {
#pragma unroll
            for (int o = 1; o < (FORM == kLong ? 32 : FORM); o *= 2)
                if constexpr (std::is_same<T, float>::value && K % 2 == 0) {
#pragma unroll
                    for (int k = 0; k < K; k += 2) {
                        const float2 t = add(make_float2(s[k], s[k + 1]), make_float2(__shfl_xor_sync(0xffffffffu, s[k], o), __shfl_xor_sync(0xffffffffu, s[k + 1], o)));
                        s[k] = t.x, s[k + 1] = t.y;
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < K; ++k) s[k] += __shfl_xor_sync(0xffffffffu, s[k], o);
                }
        }
    }
    template <int K>
    __device__ __forceinline__ void all(float (&s)[K]) {
        over_lanes(s);
        if (WIDE) {
            float* mine = scratch + turn * 64;
            turn ^= 1;                                // in turns: one barrier a sum
            if (threadIdx.x % 32 == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) mine[threadIdx.x / 32 * K + k] = s[k];
            __syncthreads();
            Vec<float, K> of = load<float, K>(mine);
#pragma unroll
            for (int k = 0; k < K; ++k) s[k] = of.v[k];
            for (int w = 1; w < threads / 32; ++w) {
                of = load<float, K>(mine + w * K);
#pragma unroll
                for (int k = 0; k < K; ++k) s[k] += of.v[k];
            }
        }
    }
    // near the mean of a row: of a short row the mean of its first thread's values, of a long one the mean but for its rounding
    __device__ __forceinline__ void near(float (&s)[2], float inv_own, float inv_c) {
        if (WIDE) {
            all(s);
            s[0] *= inv_c, s[1] *= inv_c;
        } else {
            const int first = threadIdx.x % 32 & ~(threads - 1);
            s[0] = __shfl_sync(0xffffffffu, s[0] * inv_own, first);
            s[1] = __shfl_sync(0xffffffffu, s[1] * inv_own, first);
        }
    }
    __device__ __forceinline__ float near(float s, float inv_own, float inv_c) {
        float v[2] = {s, 0.0f};
        near(v, inv_own, inv_c);
        return v[0];
    }
    // the same in 64 bits, of one value; every thread of the CTA calls it
    __device__ __forceinline__ double exactly(double s) {
        double v[1] = {s};
        over_lanes(v);
        s = v[0];
        if (WIDE) {
            double* mine = reinterpret_cast<double*>(scratch + turn * 64);
            turn ^= 1;
            if (threadIdx.x % 32 == 0) mine[threadIdx.x / 32] = s;
            __syncthreads();
            s = mine[0];
            for (int w = 1; w < threads / 32; ++w) s += mine[w];
        }
        return s;
    }
};

__device__ __forceinline__ float2 sum_of(const Eight& e) {
    return add(add(e.v[0], e.v[1]), add(e.v[2], e.v[3]));
}
__device__ __forceinline__ float across(float2 s) { return s.x + s.y; }
// sum of products, of the eight
__device__ __forceinline__ float dot(const Eight& p, const Eight& q) {
    return across(fma(p.v[0], q.v[0], fma(p.v[1], q.v[1], fma(p.v[2], q.v[2], mul(p.v[3], q.v[3])))));
}
// e - mean at the row's channels, 0 beyond
template <int V>
__device__ __forceinline__ void centre(Eight& e, float mean, int lane, const BlockArgs& a) {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) e.v[i] = add(e.v[i], both(-mean));
    if (a.ragged)
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            if (!inside<V>(lane, a, 2 * i)) e.v[i].x = 0.0f;
            if (!inside<V>(lane, a, 2 * i + 1)) e.v[i].y = 0.0f;
        }
}
// From the sums over a row of its values and of their squares -- of a layer norm, of their distances from a value near the
// mean: v^ = root v + shift.  The first thread's mean is near enough: its square from the mean is at most a thread's
// share of the row's sum of squares, so that the difference loses at most five bits in rows of 256 channels, and with
// values in no special order none.  A row of equal values is 0, and one far from zero keeps its spread.  A row with a NaN is
// NaN throughout, and so is a layer norm's with an infinity; by its root mean square the rest of that row is 0.
struct Scaling {
    float root, shift;
    __device__ __forceinline__ Scaling(int kind, float total, float square, const BlockArgs& a) {
        const float left = kind == PP_NORM_LAYER ? total * a.inv_c : 0.0f;
        root = kind == PP_NORM_NONE ? 1.0f : rsqrtf(larger(fmaf(-left, left, square * a.inv_c), 0.0f) + a.eps);
        shift = -left * root;
    }
};

struct At {
    int sample, pixel;
};
__device__ __forceinline__ At at_row(int row, const BlockArgs& a) {
    const int n = a.pixels == 1 ? row : (int)((uint64_t)(uint32_t)row * a.pixels_mul >> a.pixels_shift);
    return {n, row - n * (int)a.pixels};
}
// the same, or, where every tensor's samples follow one another as its pixels do, all as one sample
__device__ __forceinline__ At place_of(int row, const BlockArgs& a) { return a.flat ? At{0, row} : at_row(row, a); }
// Where a thread's channels of a row are: of a dense tensor so many from the CTA's first row on, of others by their strides.
struct Spot {
    At at;
    int64_t begin;                                    // (dense) the CTA's first row: the same for all threads
    uint32_t offset;
};
template <bool DENSE, typename T>
__device__ __forceinline__ const T* spot_in(const void* p, const Spot& s, int64_t pixel, int64_t sample, int lane_first) {
    if (DENSE) return static_cast<const T*>(p) + s.begin + s.offset;
    return static_cast<const T*>(p) + s.at.sample * sample + (int64_t)s.at.pixel * (int)pixel + lane_first;
}

__device__ __forceinline__ float act_of(float z, int act) {
    if (act == PP_ACT_RELU) return larger(z, 0.0f);
    if (act == PP_ACT_SILU) return z * approx_rcp(1.0f + approx_exp2(-1.4426950408889634f * z));
    return z;
}

// -------------------------------------------------------------------------------- forward

template <typename TX, typename TB, int V, int FORM, int KIND>
__global__ void __launch_bounds__(FORM == kLong ? 512 : kBlockThreads, FORM == kLong ? 1 : 3) block_rows(BlockArgs a) {
    constexpr bool WIDE = FORM == kLong, DENSE = KIND != kStrided, FIXED = KIND == kRms || KIND == kLayer;
    const int post = FIXED ? KIND : a.post, pre = FIXED ? KIND : a.pre;
    const bool has_b = FIXED || a.b;
    extern __shared__ __align__(16) char ring[];
    __shared__ __align__(16) float scratch[WIDE ? 128 : 1];
    const int threads = FORM > 0 ? FORM : a.threads;
    const int lane = WIDE ? threadIdx.x : threadIdx.x % threads;
    const int here = WIDE ? 1 : kBlockThreads / threads, mine = WIDE ? 0 : threadIdx.x / threads;
    RowSum<FORM> sum{threads, scratch};
    using X = Ahead<TX, V>;
    using B = Ahead<TB, V>;
    // consecutive rows: the gate changes with the sample
    const int begin = blockIdx.x * a.stretch, end = min(a.rows, begin + a.stretch);
    const uint32_t stride = (uint32_t)(here * a.C);
    const int64_t begin_at = (int64_t)begin * a.C;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    const int round = (X::kBytes + B::kBytes) * blockDim.x, b_at = X::kBytes * blockDim.x;
    const auto spot_of = [&](int row, bool there, uint32_t offset) { return Spot{DENSE ? At{0, 0} : place_of(there ? row : 0, a), begin_at, offset}; };
    const auto x_in = [&](const Spot& s) { return spot_in<DENSE, TX>(a.x, s, a.x_pixel, a.x_sample, lane * V); };
    const auto b_in = [&](const Spot& s) { return spot_in<DENSE, TB>(a.b, s, a.b_pixel, a.b_sample, lane * V); };
    const bool in_row = lane < a.vectors;             // (V = 8)
    const auto live_if = [&](bool there) {
        return [=, &a](int k) { return there && (V == 8 ? in_row : lane + k * threads < a.vectors); };
    };
    const auto ask = [&](int base, uint32_t offset, int slot) {
        if (base < end) {
            const bool there = base + mine < end;
            const Spot s = spot_of(base + mine, there, offset);
            X::ask(ring_at + slot * round, x_in(s), threads, live_if(there));
            if (has_b) B::ask(ring_at + slot * round + b_at, b_in(s), threads, live_if(there));
        }
        copies_end();
    };
    uint32_t offset = (uint32_t)(mine * a.C + lane * V);
    for (int k = 0; k < kRounds - 1; ++k) ask(begin + k * here, offset + k * stride, k);

    // the block's weight and bias with the residual scale in them, the stream's
    __shared__ __align__(16) float shared[4][kHeldFloats<FORM>];
    Held<FORM> wb(shared[0], lane), bb(shared[1], lane), w(shared[2], lane), bias(shared[3], lane);
    {
        const Eight sc = parameter<V>(a.scale, 1.0f, lane, a);
        wb.set(times<V>(parameter<V>(a.post_weight, 1.0f, lane, a), sc), threads, mine == 0);
        bb.set(times<V>(parameter<V>(a.post_bias, 0.0f, lane, a), sc), threads, mine == 0);
        w.set(parameter<V>(a.weight, 1.0f, lane, a), threads, mine == 0);
        bias.set(parameter<V>(a.bias, 0.0f, lane, a), threads, mine == 0);
        if (!WIDE) __syncthreads();
    }
    Eight gate = parameter<V>(nullptr, 1.0f, lane, a);
    int gate_of = -1;
    const float inv_own = 1.0f / own_channels<V>(lane, a);
    int slot = 0;
    for (int base = begin; base < end; base += here, offset += stride) {
        const int row = base + mine;
        const bool there = row < end;
        ask(base + (kRounds - 1) * here, offset + (kRounds - 1) * stride, slot == 0 ? kRounds - 1 : slot - 1);   // where the round before has read
        copies_wait<kRounds - 1>();
        const uint32_t place = ring_at + slot * round;
        slot = slot == kRounds - 1 ? 0 : slot + 1;
        const auto live = live_if(there);
        const Spot at = spot_of(row, there, offset);
        if (a.gate) {
            const int sample = at_row(there ? row : 0, a).sample;
            if (there && sample != gate_of) {
                gate = parameter<V>(a.gate + (int64_t)sample * a.C, 1.0f, lane, a);
                gate_of = sample;
            }
        }
        Eight h = widened(X::get(place, x_in(at), threads, live));
        if (has_b) {
            Eight b = widened(B::get(place + b_at, b_in(at), threads, live));
            if (post == PP_NORM_LAYER) centre<V>(b, sum.near(across(sum_of(b)), inv_own, a.inv_c), lane, a);
            float q[2] = {post == PP_NORM_LAYER ? across(sum_of(b)) : 0.0f, dot(b, b)};
            if (post != PP_NORM_NONE) sum.all(q);
            const Scaling r(post, q[0], q[1], a);
            const Eight pw = wb.get(threads), pb = bb.get(threads);
#pragma unroll
            for (int i = 0; i < E / 2; ++i)
                h.v[i] = fma(fma(fma(b.v[i], both(r.root), both(r.shift)), pw.v[i], pb.v[i]), gate.v[i], h.v[i]);
            const Raw<TX, V> out = narrowed<TX, V>(h);
            put(static_cast<TX*>(a.h) + begin_at + offset, out, threads, live);
            h = widened(out);                         // the second norm is of the stream as it is stored
        }
        if (pre == PP_NORM_NONE) continue;
        if (pre == PP_NORM_LAYER) centre<V>(h, sum.near(across(sum_of(h)), inv_own, a.inv_c), lane, a);
        float q[2] = {pre == PP_NORM_LAYER ? across(sum_of(h)) : 0.0f, dot(h, h)};
        sum.all(q);
        const Scaling r(pre, q[0], q[1], a);
        const Eight nw = w.get(threads), nb = bias.get(threads);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) h.v[i] = fma(fma(h.v[i], both(r.root), both(r.shift)), nw.v[i], nb.v[i]);
        if (a.act != PP_ACT_NONE)
#pragma unroll
            for (int i = 0; i < E / 2; ++i) h.v[i] = make_float2(act_of(h.v[i].x, a.act), act_of(h.v[i].y, a.act));
        put(static_cast<TB*>(a.y) + begin_at + offset, narrowed<TB, V>(h), threads, live);
    }
}

// -------------------------------------------------------------------------------- backward

// Whether z = w (h - mean) r + bias is above 0, where fp32 cannot tell: mean and root in 64 bits.  Every thread of the CTA
// (kLong) or of the warp calls it; value(k) is the thread's k-th channel's.  One channel at a time: it is rarely come to, and
// is to take few registers from what is.
template <int V, int FORM, typename F>
__device__ __forceinline__ unsigned above_zero(F&& value, const BlockArgs& a, int lane, RowSum<FORM>& sum) {
    double mean = 0, square = 0;
    if (a.pre == PP_NORM_LAYER) {
#pragma unroll 1
        for (int k = 0; k < E; ++k) mean += (double)value(k);            // beyond the row they are 0
        mean = sum.exactly(mean) / a.C;
    }
#pragma unroll 1
    for (int k = 0; k < E; ++k)
        if (inside<V>(lane, a, k)) square += ((double)value(k) - mean) * ((double)value(k) - mean);
    const double r = 1.0 / sqrt(sum.exactly(square) / a.C + (double)a.eps);
    unsigned above = 0;
#pragma unroll 1
    for (int k = 0; k < E; ++k) {
        const int c = channel<V>(lane, sum.threads, k);
        if (c >= a.C) continue;
        const double z = ((double)value(k) - mean) * r * (a.weight ? (double)a.weight[c] : 1.0) + (a.bias ? (double)a.bias[c] : 0.0);
        above |= (unsigned)(z > 0) << k;
    }
    return above;
}

template <typename TX, typename TB, int V, int FORM, int KIND>
__global__ void __launch_bounds__(FORM == kLong ? 512 : kBlockBackThreads, FORM == kLong ? 1 : 4) block_back_rows(BlockArgs a) {
    constexpr bool WIDE = FORM == kLong, DENSE = KIND != kStrided, FIXED = KIND == kRms || KIND == kLayer;
    constexpr int R = kRoundsBack<TX, TB, WIDE>;
    extern __shared__ __align__(16) char ring[];
    __shared__ __align__(16) float scratch[WIDE ? 128 : 1];
    __shared__ float lanes_sum[WIDE ? 1 : 2 * kBlockBackThreads * E];
    const int threads = FORM > 0 ? FORM : a.threads;
    const int lane = WIDE ? threadIdx.x : threadIdx.x % threads;
    const int here = WIDE ? 1 : kBlockBackThreads / threads, mine = WIDE ? 0 : threadIdx.x / threads;
    RowSum<FORM> sum{threads, scratch};
    const int post_kind = FIXED ? KIND : a.post, pre_kind = FIXED ? KIND : a.pre;
    const bool pre = pre_kind != PP_NORM_NONE, post = post_kind != PP_NORM_NONE, has_b = FIXED || a.b, has_dh = FIXED || a.dh;
    __shared__ __align__(16) float shared[3][kHeldFloats<FORM>];
    Held<FORM> w_held(shared[0], lane), bias_held(shared[1], lane), k_held(shared[2], lane);
    using X = Ahead<TX, V>;
    using B = Ahead<TB, V>;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    const int x_bytes = X::kBytes * blockDim.x, b_bytes = B::kBytes * blockDim.x, round = 2 * (x_bytes + b_bytes);
    const int d_at = 0, h_at = x_bytes, y_at = 2 * x_bytes, b_at = y_at + b_bytes;
    const int begin = blockIdx.x * a.stretch, end = min(a.rows, begin + a.stretch);
    const int64_t begin_at = (int64_t)begin * a.C;
    const auto spot_of = [&](int row, uint32_t offset) { return Spot{DENSE ? At{0, 0} : place_of(row, a), begin_at, offset}; };
    const auto h_in = [&](const Spot& s) { return spot_in<DENSE, TX>(a.x, s, a.x_pixel, a.x_sample, lane * V); };
    const auto b_in = [&](const Spot& s) { return spot_in<DENSE, TB>(a.b, s, a.b_pixel, a.b_sample, lane * V); };
    const auto d_in = [&](const Spot& s) { return spot_in<DENSE, TX>(a.dh, s, a.dh_pixel, a.dh_sample, lane * V); };
    const auto y_in = [&](const Spot& s) { return spot_in<DENSE, TB>(a.dy, s, a.dy_pixel, a.dy_sample, lane * V); };
    const bool in_row = lane < a.vectors;             // (V = 8)
    const auto live_if = [&](bool there) {
        return [=, &a](int k) { return there && (V == 8 ? in_row : lane + k * threads < a.vectors); };
    };
    // asks for a round of rows, `last` the end of their sample's
    const auto ask = [&](int base, int last, uint32_t offset, int slot) {
        if (base < last) {
            const bool there = base + mine < last;
            const Spot s = spot_of(there ? base + mine : base, offset);
            const auto live = live_if(there);
            const uint32_t place = ring_at + slot * round;
            if (pre) X::ask(place + h_at, h_in(s), threads, live);
            if (has_b) B::ask(place + b_at, b_in(s), threads, live);
            if (pre) B::ask(place + y_at, y_in(s), threads, live);
            if (has_dh) X::ask(place + d_at, d_in(s), threads, live);
        }
        copies_end();
    };

    // a sample's rows of this CTA, the first ones asked for (with a gate; without one all rows are as of one sample)
    const uint32_t stride = (uint32_t)(here * a.C);
    At start;
    int to = end;
    uint32_t offset;
    const auto enter = [&](int from) {
        start = at_row(from, a);
        if (a.gate) to = min(end, from - start.pixel + (int)a.pixels);     // (a row of the sample plus its pixels may pass 2^31)
        offset = (uint32_t)((from - begin + mine) * a.C + lane * V);
        for (int k = 0; k < R - 1; ++k) ask(from + k * here, to, offset + k * stride, k);
    };
    enter(begin);

    const Eight zero{};
    const float inv_own = 1.0f / own_channels<V>(lane, a);
    float reach = 0;                                  // how near to 0 a z of this thread's may be without its sign being sure
    {
        const Eight w = parameter<V>(a.weight, 1.0f, lane, a);
        Eight bias = parameter<V>(a.bias, 0.0f, lane, a);
#pragma unroll
        for (int i = 0; i < E / 2; ++i)
            reach = fmaxf(reach, fmaxf(fmaf(fabsf(w.v[i].x), sqrtf((float)a.C) + 1.0f, fabsf(bias.v[i].x)),
                                       fmaf(fabsf(w.v[i].y), sqrtf((float)a.C) + 1.0f, fabsf(bias.v[i].y))));
        reach *= 3.8147e-6f;
        w_held.set(w, threads, mine == 0);
#pragma unroll
        for (int i = 0; i < E; ++i)                   // (beyond the row z is 1, and its sign sure)
            if (!inside<V>(lane, a, i)) reinterpret_cast<float*>(bias.v)[i] = 1.0f;
        bias_held.set(bias, threads, mine == 0);
    }
    // where the rows' threads leave channel c's sums: by the thread's number of it, then by threads
    const auto place_in_sums = [&](int c) {
        const int vector = c / V, turn = vector / threads;
        return (turn * V + c % V) * threads + vector - turn * threads;
    };
    // the means over a row of t (of a layer norm) and of t v^
    const auto means = [&](int kind, const Eight& t, const Eight& v) {
        float q[2] = {kind == PP_NORM_LAYER ? across(sum_of(t)) : 0.0f, dot(t, v)};
        sum.all(q);
        return make_float2(q[0] * a.inv_c, q[1] * a.inv_c);
    };
    Eight s_w = zero, s_b = zero, s_e = zero, s_f = zero;        // sums of dz h^, dz, and of a sample dh b^, dh
    // the sums over all samples, in shared memory: of post_weight, post_bias and scale, thread c's, and so on (WIDE: the thread's eight channels')
    constexpr int OWN = WIDE ? E : 32 * E / kBlockBackThreads;
    float* totals = reinterpret_cast<float*>(ring + R * 2 * (Ahead<TX, V>::kBytes + Ahead<TB, V>::kBytes) * blockDim.x) + threadIdx.x;
    const auto total = [&](int which, int i) -> float& { return totals[(which * OWN + i) * blockDim.x]; };
#pragma unroll
    for (int i = 0; i < 3 * OWN; ++i) total(0, i) = 0.0f;

    for (int from = begin; from < end;) {
        const float* gate = a.gate ? a.gate + (int64_t)start.sample * a.C : nullptr;
        // what dh is multiplied with on its way to the normalised block
        if (!WIDE) __syncthreads();                   // (the sample before has been summed)
        k_held.set(times<V>(parameter<V>(a.post_weight, 1.0f, lane, a), times<V>(parameter<V>(a.scale, 1.0f, lane, a), parameter<V>(gate, 1.0f, lane, a))),
                   threads, mine == 0);
        if (!WIDE) __syncthreads();

        int slot = 0;
        for (int base = from; base < to; base += here, offset += stride) {
            const int row = base + mine;
            const bool there = row < to;
            ask(base + (R - 1) * here, to, offset + (R - 1) * stride, slot == 0 ? R - 1 : slot - 1);
            copies_wait<R - 1>();
            const uint32_t place = ring_at + slot * round;
            slot = slot == R - 1 ? 0 : slot + 1;
            const auto live = live_if(there);
            const Spot at = spot_of(there ? row : base, offset);
            Eight h = zero, b = zero;
            if (pre) h = widened(X::get(place + h_at, h_in(at), threads, live));
            if (has_b) b = widened(B::get(place + b_at, b_in(at), threads, live));
            // both norms
            float centres[2] = {0, 0};
            if (pre_kind == PP_NORM_LAYER || post_kind == PP_NORM_LAYER) {
                centres[0] = across(sum_of(h)), centres[1] = across(sum_of(b));
                sum.near(centres, inv_own, a.inv_c);
            }
            if (pre_kind == PP_NORM_LAYER) centre<V>(h, centres[0], lane, a);
            if (post_kind == PP_NORM_LAYER) centre<V>(b, centres[1], lane, a);
            float moments[4] = {pre_kind == PP_NORM_LAYER ? across(sum_of(h)) : 0.0f, post_kind == PP_NORM_LAYER ? across(sum_of(b)) : 0.0f, dot(h, h), dot(b, b)};
            if (pre || post) sum.all(moments);
            const Scaling sh(pre_kind, moments[0], moments[2], a), sb(post_kind, moments[1], moments[3], a);
            const float2 r = there ? make_float2(sh.root, sb.root) : make_float2(0.0f, 0.0f);
            const float2 shift = there ? make_float2(sh.shift, sb.shift) : make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < E / 2; ++i)
                h.v[i] = fma(h.v[i], both(r.x), both(shift.x)), b.v[i] = fma(b.v[i], both(r.y), both(shift.y));
            Eight d = zero;
            if (!pre && has_dh) d = widened(X::get(place + d_at, d_in(at), threads, live));
            if (pre) {
                const Eight w = w_held.get(threads);
                Eight dz = widened(B::get(place + y_at, y_in(at), threads, live));
                if (a.act == PP_ACT_RELU) {
                    // fp32's z is off by less than 2^-18 of its terms' sizes (each value, the mean, and the root by some 16 roundings
                    // of the row's sums), |h^| is at most the root of C: where the smallest z is nearer to 0 than that, and then
                    // some z than its own terms allow, the signs are taken in 64 bits
                    const Eight bias = bias_held.get(threads);
                    float2 z[E / 2];
                    float least = INFINITY;
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) {
                        z[i] = fma(h.v[i], w.v[i], bias.v[i]);
                        least = fminf(least, fminf(fabsf(z[i].x), fabsf(z[i].y)));
                    }
                    const float spread = 1.0f + 2.0f * fabsf(pre_kind == PP_NORM_LAYER ? centres[0] * r.x : 0.0f);
                    bool close = there && least <= reach * spread;
                    if (close) {                      // more closely, of each value by itself
                        const float* zf = reinterpret_cast<const float*>(z);
                        const float* hf = reinterpret_cast<const float*>(h.v);
                        const float* wf = reinterpret_cast<const float*>(w.v);
                        const float* bf = reinterpret_cast<const float*>(bias.v);
                        close = false;
#pragma unroll
                        for (int i = 0; i < E; ++i)
                            close = close || fabsf(zf[i]) <= 3.8147e-6f * fmaf(fabsf(wf[i]), fabsf(hf[i]) + spread, fabsf(bf[i]));
                    }
                    if (WIDE ? __syncthreads_or(close) : __any_sync(0xffffffffu, close)) {
                        const unsigned above = above_zero<V, FORM>([&](int k) { return there && inside<V>(lane, a, k) ? X::one(place + h_at, h_in(at), threads, k) : 0.0f; }, a, lane, sum);
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) {
                            if (!(above >> (2 * i) & 1)) dz.v[i].x = 0.0f;
                            if (!(above >> (2 * i + 1) & 1)) dz.v[i].y = 0.0f;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) {
                            if (!(z[i].x > 0.0f)) dz.v[i].x = 0.0f;
                            if (!(z[i].y > 0.0f)) dz.v[i].y = 0.0f;
                        }
                    }
                } else if (a.act == PP_ACT_SILU) {
                    const Eight bias = bias_held.get(threads);
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) {
                        const float2 z = fma(h.v[i], w.v[i], bias.v[i]);
                        const float sx = approx_rcp(1.0f + approx_exp2(-1.4426950408889634f * z.x));
                        const float sy = approx_rcp(1.0f + approx_exp2(-1.4426950408889634f * z.y));
                        dz.v[i] = mul(dz.v[i], make_float2(fmaf(z.x * sx, 1.0f - sx, sx), fmaf(z.y * sy, 1.0f - sy, sy)));
                    }
                }
                Eight t;
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    s_w.v[i] = fma(dz.v[i], h.v[i], s_w.v[i]);
                    s_b.v[i] = add(dz.v[i], s_b.v[i]);
                    t.v[i] = mul(dz.v[i], w.v[i]);
                }
                const float2 q = means(pre_kind, t, h);
                if (has_dh) d = widened(X::get(place + d_at, d_in(at), threads, live));
#pragma unroll
                for (int i = 0; i < E / 2; ++i)
                    d.v[i] = fma(fma(h.v[i], both(-q.y), add(t.v[i], both(-q.x))), both(r.x), d.v[i]);
            }
            put(static_cast<TX*>(a.dx) + begin_at + offset, narrowed<TX, V>(d), threads, live);
            if (!has_b) continue;
            const Eight k = k_held.get(threads);
            Eight t;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                s_e.v[i] = fma(d.v[i], b.v[i], s_e.v[i]);     // (of no row d is 0)
                s_f.v[i] = add(d.v[i], s_f.v[i]);
                t.v[i] = mul(d.v[i], k.v[i]);
            }
            if (post) {
                const float2 q = means(post_kind, t, b);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) t.v[i] = mul(fma(b.v[i], both(-q.y), add(t.v[i], both(-q.x))), both(r.y));
            }
            put(static_cast<TB*>(a.db) + begin_at + offset, narrowed<TB, V>(t), threads, live);
        }

        const bool first = from == begin, last = to == end;
        const bool whole = (first ? start.pixel == 0 : true) && (last ? at_row(end - 1, a).pixel == a.pixels - 1 : true);
        const int64_t sample = start.sample;
        from = to;
        if (!last) enter(to);

        // the sample's sums: of the block's norm, the gate and the scale
        if (has_b) {
            float* e_all = lanes_sum;
            float* f_all = lanes_sum + kBlockBackThreads * E;
            if (!WIDE) {
                __syncthreads();
                const float* pe = reinterpret_cast<const float*>(s_e.v);
                const float* pf = reinterpret_cast<const float*>(s_f.v);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    e_all[(mine * E + i) * threads + lane] = pe[i];
                    f_all[(mine * E + i) * threads + lane] = pf[i];
                }
                __syncthreads();
            }
            // (all asked for before the first result is stored: the compiler cannot know that they are not the same)
            float ga[OWN], sc[OWN], pw[OWN], pb[OWN];
#pragma unroll
            for (int i = 0; i < OWN; ++i) {
                const int c = WIDE ? channel<V>(lane, threads, i) : threadIdx.x + i * kBlockBackThreads;
                const bool is = c < a.C;
                ga[i] = gate && is ? gate[c] : 1.0f, sc[i] = a.scale && is ? a.scale[c] : 1.0f;
                pw[i] = a.post_weight && is ? a.post_weight[c] : 1.0f, pb[i] = a.post_bias && is ? a.post_bias[c] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < OWN; ++i) {
                const int c = WIDE ? channel<V>(lane, threads, i) : threadIdx.x + i * kBlockBackThreads;
                if (c >= a.C) continue;
                float e = 0, f = 0;
                if (WIDE) {
                    e = reinterpret_cast<const float*>(s_e.v)[i];
                    f = reinterpret_cast<const float*>(s_f.v)[i];
                } else {
                    const int at = place_in_sums(c);
                    for (int g = 0; g < here; ++g) e += e_all[g * threads * E + at], f += f_all[g * threads * E + at];
                }
                const float joined = fmaf(pw[i], e, a.post_bias ? pb[i] * f : 0.0f);
                total(0, i) = fmaf(sc[i] * ga[i], e, total(0, i));
                total(1, i) = fmaf(sc[i] * ga[i], f, total(1, i));
                total(2, i) = fmaf(ga[i], joined, total(2, i));
                if (a.dgate) {
                    if (whole)
                        a.dgate[sample * a.C + c] = sc[i] * joined;
                    else
                        a.gates[((int64_t)blockIdx.x * 2 + !first) * a.C + c] = sc[i] * joined;
                }
            }
            s_e = s_f = zero;
        }
    }

    // the CTA's sums
    float* out = a.sums + (int64_t)blockIdx.x * kBlockSums * a.C;
    if (!WIDE) {
        __syncthreads();
        const float* pw = reinterpret_cast<const float*>(s_w.v);
        const float* pb = reinterpret_cast<const float*>(s_b.v);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            lanes_sum[(mine * E + i) * threads + lane] = pw[i];
            lanes_sum[kBlockBackThreads * E + (mine * E + i) * threads + lane] = pb[i];
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int c = WIDE ? channel<V>(lane, threads, i) : threadIdx.x + i * kBlockBackThreads;
        if (c >= a.C) continue;
        float e = 0, f = 0;
        if (WIDE) {
            e = reinterpret_cast<const float*>(s_w.v)[i];
            f = reinterpret_cast<const float*>(s_b.v)[i];
        } else {
            const int at = place_in_sums(c);
            for (int g = 0; g < here; ++g) e += lanes_sum[g * threads * E + at], f += lanes_sum[kBlockBackThreads * E + g * threads * E + at];
        }
        out[c] = e;
        out[a.C + c] = f;
#pragma unroll
        for (int k = 0; k < 3; ++k) out[(2 + k) * a.C + c] = total(k, i);
    }
}

// more shared memory than a launch has by itself: once for each kernel and device
template <typename K>
cudaError_t allow_shared(K* kernel, std::atomic<uint64_t>& done, size_t bytes) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev >= 64 || !(done.load(std::memory_order_relaxed) >> dev & 1))) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e == cudaSuccess && dev < 64) done.fetch_or(uint64_t(1) << dev);
    }
    if (e != cudaSuccess) cudaGetLastError();
    return e;
}
template <typename TX, typename TB, int V, int FORM, int KIND>
cudaError_t forward_rows(const BlockArgs& a, cudaStream_t st) {
    constexpr int kRound = Ahead<TX, V>::kBytes + Ahead<TB, V>::kBytes, kMost = FORM == kLong ? 512 : kBlockThreads;
    static std::atomic<uint64_t> allowed{0};
    if (const cudaError_t e = allow_shared(block_rows<TX, TB, V, FORM, KIND>, allowed, kRounds * kRound * kMost)) return e;
    const int threads = FORM == kLong ? a.threads : kBlockThreads, here = threads / a.threads;
    int each = 3;                                     // CTAs of an SM: one wave, so of long rows what fits (32 x 512 x 28 x 28 takes 29 us, 40 with a
    if (FORM == kLong) {                              // sixth of the CTAs left for a second one)
        static std::atomic<int> fit[16];
        std::atomic<int>& f = fit[threads / 32 - 1];
        if (!(each = f.load(std::memory_order_relaxed))) {
            if (const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, block_rows<TX, TB, V, FORM, KIND>, threads, kRounds * kRound * threads)) {
                cudaGetLastError();
                return e;
            }
            f = each = std::max(1, each);
        }
    }
    const int most = 152 * each, rounds = (a.rows + here - 1) / here;
    BlockArgs b = a;
    b.stretch = (rounds + most - 1) / most * here;
    block_rows<TX, TB, V, FORM, KIND><<<(a.rows + b.stretch - 1) / b.stretch, threads, kRounds * kRound * threads, st>>>(b);
    return cudaGetLastError();
}
template <typename TX, typename TB, int V, int FORM, int KIND>
cudaError_t backward_rows(const BlockArgs& a, cudaStream_t st) {
    constexpr int kEach = kRoundsBack<TX, TB, FORM == kLong> * 2 * (Ahead<TX, V>::kBytes + Ahead<TB, V>::kBytes) +
                          3 * (FORM == kLong ? E : 32 * E / kBlockBackThreads) * (int)sizeof(float);      // of a thread
    static std::atomic<uint64_t> allowed{0};
    if (const cudaError_t e = allow_shared(block_back_rows<TX, TB, V, FORM, KIND>, allowed, kEach * (FORM == kLong ? 512 : kBlockBackThreads))) return e;
    const int threads = FORM == kLong ? a.threads : kBlockBackThreads;
    block_back_rows<TX, TB, V, FORM, KIND><<<a.ctas, threads, kEach * threads, st>>>(a);
    if (const cudaError_t e = cudaGetLastError()) return e;
    return block_join(a, st);
}
// f with the form of the kernels that a call takes, and with the kind of its norms where that goes with it
template <int V, typename F>
cudaError_t by_form(const BlockArgs& a, F&& f) {
    using std::integral_constant;
    const auto of_kind = [&](auto form) {
        if (a.pre != a.post || a.pre == PP_NORM_NONE || !a.full) return f(form, integral_constant<int, kDense>());
        return a.pre == PP_NORM_RMS ? f(form, integral_constant<int, kRms>()) : f(form, integral_constant<int, kLayer>());
    };
    if (a.threads > 32) {
        if constexpr (V > 1)
            if (a.dense) return of_kind(integral_constant<int, kLong>());
        return f(integral_constant<int, kLong>(), integral_constant<int, kStrided>());
    }
    if constexpr (V > 1)
        if (a.dense) {
            if (a.threads >= 8)
                return a.threads == 32   ? of_kind(integral_constant<int, 32>())
                       : a.threads == 16 ? of_kind(integral_constant<int, 16>())
                                         : of_kind(integral_constant<int, 8>());
            const integral_constant<int, kDense> any;
            return a.threads == 4 ? f(integral_constant<int, 4>(), any) : a.threads == 2 ? f(integral_constant<int, 2>(), any) : f(integral_constant<int, 1>(), any);
        }
    return f(integral_constant<int, kShort>(), integral_constant<int, kStrided>());
}
template <typename TX, typename TB, int V>
cudaError_t forward_as(const BlockArgs& a, cudaStream_t st) {
    return by_form<V>(a, [&](auto form, auto kind) { return forward_rows<TX, TB, V, decltype(form)::value, decltype(kind)::value>(a, st); });
}
template <typename TX, typename TB, int V>
cudaError_t backward_as(const BlockArgs& a, cudaStream_t st) {
    return by_form<V>(a, [&](auto form, auto kind) { return backward_rows<TX, TB, V, decltype(form)::value, decltype(kind)::value>(a, st); });
}

}  // namespace

template <typename TX, typename TB>
cudaError_t BlockKernels<TX, TB>::forward(const BlockArgs& a, int V, cudaStream_t st) {
    constexpr int W = sizeof(TX) == 2 ? 8 : 4;
    return V == W ? forward_as<TX, TB, W>(a, st) : V == 2 ? forward_as<TX, TB, 2>(a, st) : forward_as<TX, TB, 1>(a, st);
}
template <typename TX, typename TB>
cudaError_t BlockKernels<TX, TB>::backward(const BlockArgs& a, int V, cudaStream_t st) {
    constexpr int W = sizeof(TX) == 2 ? 8 : 4;
    return V == W ? backward_as<TX, TB, W>(a, st) : V == 2 ? backward_as<TX, TB, 2>(a, st) : backward_as<TX, TB, 1>(a, st);
}

}  // namespace patconv
