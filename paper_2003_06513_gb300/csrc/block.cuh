// Kernels of block.cu, for one type of blocks each in block_f32.cu, block_f16.cu and block_bf16.cu, the stream being of
// the same type or fp32.
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
    static constexpr int S = sizeof(T) * V > 16 ? 16 : sizeof(T) * V, P = E * (int)sizeof(T) / S;
    static constexpr bool kAsync = S >= 4;
    static constexpr int kBytes = kAsync ? E * (int)sizeof(T) : 0;       // of a thread and round
    // bytes from the row's first channel to piece k, and whether the row has it
    static __device__ __forceinline__ int64_t offset(int lane, const BlockArgs& a, int k) {
        return sizeof(T) * V > 16 ? (int64_t)lane * V * sizeof(T) + k * S : (int64_t)(lane + k * a.threads) * S;
    }
    static __device__ __forceinline__ bool has(int lane, const BlockArgs& a, int k) {
        return (sizeof(T) * V > 16 ? lane : lane + k * a.threads) < a.vectors;
    }
    static __device__ __forceinline__ void ask(uint32_t place, const T* row, int lane, const BlockArgs& a, bool there) {
        if constexpr (kAsync) {
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const bool wanted = there && has(lane, a, k);
                const char* from = reinterpret_cast<const char*>(row) + (wanted ? offset(lane, a, k) : 0);
                const uint32_t to = place + (k * blockDim.x + threadIdx.x) * S;
                const int n = wanted ? S : 0;          // what is not copied becomes 0
                if constexpr (S == 16)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n) : "memory");
                else
                    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(S), "r"(n) : "memory");
            }
        }
    }
    static __device__ __forceinline__ Raw<T, V> get(const char* place, const T* row, int lane, const BlockArgs& a, bool there) {
        Raw<T, V> r;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            char* to = reinterpret_cast<char*>(&r) + k * S;
            if constexpr (kAsync) {
                Vec<char, S> v = *reinterpret_cast<const Vec<char, S>*>(place + (k * blockDim.x + threadIdx.x) * S);
                memcpy(to, &v, S);
            } else {
                T v = T(0.0f);
                if (there && has(lane, a, k)) v = row[lane + k * a.threads];
                memcpy(to, &v, S);
            }
        }
        return r;
    }
};
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
constexpr int kRounds = 4;                            // of rows that a CTA has under way, and in the backward pass; two there
template <typename TX, typename TB, bool WIDE>        // where 512 threads with all of it in fp32 would take more than there is
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
template <typename T, int V>
__device__ __forceinline__ void put(T* row, const Raw<T, V>& r, int lane, const BlockArgs& a, bool there) {
#pragma unroll
    for (int j = 0; j < E / V; ++j) {
        const int at = lane + j * a.threads;
        if (!there || at >= a.vectors) continue;
        T* p = row + (int64_t)at * V;
        if constexpr (sizeof(T) * V > 16) {
            float4 lo, hi;
            memcpy(&lo, &r.v[j], 16);
            memcpy(&hi, &r.v[j].v[4], 16);
            __stcs(reinterpret_cast<float4*>(p), lo);
            __stcs(reinterpret_cast<float4*>(p) + 1, hi);
        } else {
            store<T, V>(p, r.v[j]);
        }
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
// whether each of the eight is one of the row's channels
template <int V>
__device__ __forceinline__ bool inside(int lane, const BlockArgs& a, int k) { return lane + k / V * a.threads < a.vectors; }

// Sums over a row's threads, to all of them, in a fixed order.  WIDE: the CTA is one row's.
template <bool WIDE>
struct RowSum {
    int threads;
    float2* scratch;                                  // WIDE: 2 x 32
    int turn = 0;
    template <int K>
    __device__ __forceinline__ void all(float2 (&s)[K]) {
        const int span = WIDE ? 32 : threads;
        for (int o = 1; o < span; o *= 2)
#pragma unroll
            for (int k = 0; k < K; ++k)
                s[k] = add(s[k], make_float2(__shfl_xor_sync(0xffffffffu, s[k].x, o), __shfl_xor_sync(0xffffffffu, s[k].y, o)));
        if (WIDE) {
            float2* mine = scratch + turn * 32;
            turn ^= 1;                                // in turns: one barrier a sum
            if (threadIdx.x % 32 == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) mine[threadIdx.x / 32 * K + k] = s[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) s[k] = mine[k];
            for (int w = 1; w < threads / 32; ++w)
#pragma unroll
                for (int k = 0; k < K; ++k) s[k] = add(s[k], mine[w * K + k]);
        }
    }
    __device__ __forceinline__ float2 operator()(float2 s) {
        float2 v[1] = {s};
        all(v);
        return v[0];
    }
    __device__ __forceinline__ float operator()(float s) { return (*this)(make_float2(s, 0.0f)).x; }
    // the same in 64 bits, of one value; every thread of the CTA calls it
    __device__ __forceinline__ double exactly(double s) {
        const int span = WIDE ? 32 : threads;
        for (int o = 1; o < span; o *= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (WIDE) {
            double* mine = reinterpret_cast<double*>(scratch + turn * 32);
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
    for (int i = 0; i < E / 2; ++i) {
        e.v[i] = add(e.v[i], both(-mean));
        if (!inside<V>(lane, a, 2 * i)) e.v[i].x = 0.0f;
        if (!inside<V>(lane, a, 2 * i + 1)) e.v[i].y = 0.0f;
    }
}
// From the sums over a row of what was centred (or, of a norm by the root of the mean square, of the values) and of its squares:
// v^ = root v + shift.  The mean that was taken out is off by its own rounding, which here comes out too: a row of equal
// values is 0, and one far from zero keeps its spread.
struct Scaling {
    float root, shift;
    __device__ __forceinline__ Scaling(int kind, float total, float square, const BlockArgs& a) {
        const float left = kind == PP_NORM_LAYER ? total * a.inv_c : 0.0f;
        root = kind == PP_NORM_NONE ? 1.0f : rsqrtf(fmaf(-left, left, fmaf(square, a.inv_c, a.eps)));
        shift = kind == PP_NORM_LAYER ? -left * root : 0.0f;
    }
};

struct At {
    int sample, pixel;
};
__device__ __forceinline__ At at_row(int row, const BlockArgs& a) {
    const int n = a.pixels == 1 ? row : (int)((uint64_t)(uint32_t)row * a.pixels_mul >> a.pixels_shift);
    return {n, row - n * (int)a.pixels};
}
template <typename T>
__device__ __forceinline__ const T* row_of(const void* p, At at, int64_t pixel, int64_t sample) {
    return static_cast<const T*>(p) + at.sample * sample + at.pixel * pixel;
}
template <typename T>
__device__ __forceinline__ T* dense_row(void* p, int row, const BlockArgs& a) {
    return static_cast<T*>(p) + (int64_t)row * a.C;
}

__device__ __forceinline__ float act_of(float z, int act) {
    if (act == PP_ACT_RELU) return z != z ? z : fmaxf(z, 0.0f);
    if (act == PP_ACT_SILU) return z * approx_rcp(1.0f + approx_exp2(-1.4426950408889634f * z));
    return z;
}

// -------------------------------------------------------------------------------- forward

template <typename TX, typename TB, int V, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 512 : kBlockThreads, WIDE ? 1 : 3) block_rows(BlockArgs a) {
    extern __shared__ __align__(16) char ring[];
    __shared__ float2 scratch[WIDE ? 64 : 1];
    const int lane = WIDE ? threadIdx.x : threadIdx.x % a.threads;
    const int here = WIDE ? 1 : kBlockThreads / a.threads, mine = WIDE ? 0 : threadIdx.x / a.threads;
    RowSum<WIDE> sum{a.threads, scratch};
    // the block's weight and bias with the residual scale in them, the stream's
    Eight wb = parameter<V>(a.post_weight, 1.0f, lane, a), bb = parameter<V>(a.post_bias, 0.0f, lane, a);
    const Eight sc = parameter<V>(a.scale, 1.0f, lane, a);
    const Eight w = parameter<V>(a.weight, 1.0f, lane, a), bias = parameter<V>(a.bias, 0.0f, lane, a);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) wb.v[i] = mul(wb.v[i], sc.v[i]), bb.v[i] = mul(bb.v[i], sc.v[i]);
    Eight gate = parameter<V>(nullptr, 1.0f, lane, a);
    int gate_of = -1;

    using X = Ahead<TX, V>;
    using B = Ahead<TB, V>;
    const int step = gridDim.x * here;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    const int round = (X::kBytes + B::kBytes) * blockDim.x, b_at = X::kBytes * blockDim.x;
    const auto ask = [&](int row, int slot) {
        if (row - mine < a.rows) {                    // (of the CTA's first row: the same for all)
            const bool there = row < a.rows;
            const At at = at_row(there ? row : 0, a);
            X::ask(ring_at + slot * round, row_of<TX>(a.x, at, a.x_pixel, a.x_sample), lane, a, there);
            if (a.b) B::ask(ring_at + slot * round + b_at, row_of<TB>(a.b, at, a.b_pixel, a.b_sample), lane, a, there);
        }
        copies_end();
    };
    for (int k = 0; k < kRounds - 1; ++k) ask(blockIdx.x * here + k * step + mine, k);
    int slot = 0;
    for (int base = blockIdx.x * here; base < a.rows; base += step) {
        const int row = base + mine;
        const bool there = row < a.rows;
        const At at = at_row(there ? row : 0, a);
        ask(row + (kRounds - 1) * step, slot == 0 ? kRounds - 1 : slot - 1);     // into the places that the round before has read
        copies_wait<kRounds - 1>();
        const char* place = ring + slot * round;
        slot = slot == kRounds - 1 ? 0 : slot + 1;
        if (a.gate && there && at.sample != gate_of) {
            gate = parameter<V>(a.gate + (int64_t)at.sample * a.C, 1.0f, lane, a);
            gate_of = at.sample;
        }
        const Raw<TX, V> rx = X::get(place, row_of<TX>(a.x, at, a.x_pixel, a.x_sample), lane, a, there);
        Eight h = widened(rx);
        if (a.b) {
            Eight b = widened(B::get(place + b_at, row_of<TB>(a.b, at, a.b_pixel, a.b_sample), lane, a, there));
            if (a.post == PP_NORM_LAYER) centre<V>(b, sum(across(sum_of(b))) * a.inv_c, lane, a);
            float2 q = make_float2(0.0f, 0.0f);
            if (a.post != PP_NORM_NONE) q = sum(make_float2(across(sum_of(b)), dot(b, b)));
            const Scaling r(a.post, q.x, q.y, a);
#pragma unroll
            for (int i = 0; i < E / 2; ++i)
                h.v[i] = fma(fma(fma(b.v[i], both(r.root), both(r.shift)), wb.v[i], bb.v[i]), gate.v[i], h.v[i]);
            const Raw<TX, V> out = narrowed<TX, V>(h);
            put(dense_row<TX>(a.h, row, a), out, lane, a, there);
            h = widened(out);                         // the second norm is of the stream as it is stored
        }
        if (a.pre == PP_NORM_NONE) continue;
        if (a.pre == PP_NORM_LAYER) centre<V>(h, sum(across(sum_of(h))) * a.inv_c, lane, a);
        const float2 q = sum(make_float2(across(sum_of(h)), dot(h, h)));
        const Scaling r(a.pre, q.x, q.y, a);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            float2 z = fma(fma(h.v[i], both(r.root), both(r.shift)), w.v[i], bias.v[i]);
            if (a.act != PP_ACT_NONE) z = make_float2(act_of(z.x, a.act), act_of(z.y, a.act));
            h.v[i] = z;
        }
        put(dense_row<TB>(a.y, row, a), narrowed<TB, V>(h), lane, a, there);
    }
}

// -------------------------------------------------------------------------------- backward

// Whether z = w (h - mean) r + bias is above 0, where fp32 cannot tell: mean and root in 64 bits.  Every thread of the CTA
// (WIDE) or of the warp calls it.
template <typename TX, int V, bool WIDE>
__device__ __noinline__ unsigned above_zero(const char* place, const TX* row, bool there, const BlockArgs& a, int lane, RowSum<WIDE>& sum) {
    const Eight h = widened(Ahead<TX, V>::get(place, row, lane, a, there));
    const float* f = reinterpret_cast<const float*>(h.v);
    double mean = 0, square = 0;
    if (a.pre == PP_NORM_LAYER) {
        for (int k = 0; k < E; ++k) mean += (double)f[k];                // beyond the row they are 0
        mean = sum.exactly(mean) / a.C;
    }
    for (int k = 0; k < E; ++k)
        if (inside<V>(lane, a, k)) square += ((double)f[k] - mean) * ((double)f[k] - mean);
    const double r = 1.0 / sqrt(sum.exactly(square) / a.C + (double)a.eps);
    unsigned above = 0;
    for (int k = 0; k < E; ++k) {
        const int c = channel<V>(lane, a.threads, k);
        if (c >= a.C) continue;
        const double z = ((double)f[k] - mean) * r * (a.weight ? (double)a.weight[c] : 1.0) + (a.bias ? (double)a.bias[c] : 0.0);
        above |= (unsigned)(z > 0) << k;
    }
    return above;
}

template <typename TX, typename TB, int V, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 512 : kBlockThreads, WIDE ? 1 : 2) block_back_rows(BlockArgs a) {
    constexpr int R = kRoundsBack<TX, TB, WIDE>;
    extern __shared__ __align__(16) char ring[];
    __shared__ float2 scratch[WIDE ? 64 : 1];
    __shared__ float lanes_sum[WIDE ? 1 : 2 * kBlockThreads * E];
    const int lane = WIDE ? threadIdx.x : threadIdx.x % a.threads;
    const int here = WIDE ? 1 : kBlockThreads / a.threads, mine = WIDE ? 0 : threadIdx.x / a.threads;
    RowSum<WIDE> sum{a.threads, scratch};
    const bool pre = a.pre != PP_NORM_NONE, post = a.post != PP_NORM_NONE;
    const Eight w = parameter<V>(a.weight, 1.0f, lane, a), bias = parameter<V>(a.bias, 0.0f, lane, a);
    const Eight zero{};
    Eight s_w = zero, s_b = zero, s_e = zero, s_f = zero;        // sums of dz h^, dz, and of a sample dh b^, dh
    // the sums over all samples, in shared memory: of post_weight, post_bias and scale, thread c's (WIDE: the thread's eight channels')
    constexpr int OWN = WIDE ? E : 1;
    float* totals = reinterpret_cast<float*>(ring + R * 2 * (Ahead<TX, V>::kBytes + Ahead<TB, V>::kBytes) * blockDim.x) + threadIdx.x;
    const auto total = [&](int which, int i) -> float& { return totals[(which * OWN + i) * blockDim.x]; };
#pragma unroll
    for (int i = 0; i < 3 * OWN; ++i) total(0, i) = 0.0f;

    using X = Ahead<TX, V>;
    using B = Ahead<TB, V>;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    const int x_bytes = X::kBytes * blockDim.x, b_bytes = B::kBytes * blockDim.x, round = 2 * (x_bytes + b_bytes);
    const int d_at = 0, h_at = x_bytes, y_at = 2 * x_bytes, b_at = y_at + b_bytes;
    // asks for a round of rows, `last` the end of their sample's
    const auto ask = [&](int base, int last, int slot) {
        if (base < last) {
            const bool there = base + mine < last;
            const At at = at_row(there ? base + mine : base, a);
            const uint32_t place = ring_at + slot * round;
            if (pre) X::ask(place + h_at, row_of<TX>(a.x, at, a.x_pixel, a.x_sample), lane, a, there);
            if (a.b) B::ask(place + b_at, row_of<TB>(a.b, at, a.b_pixel, a.b_sample), lane, a, there);
            if (pre) B::ask(place + y_at, row_of<TB>(a.dy, at, a.dy_pixel, a.dy_sample), lane, a, there);
            if (a.dh) X::ask(place + d_at, row_of<TX>(a.dh, at, a.dh_pixel, a.dh_sample), lane, a, there);
        }
        copies_end();
    };

    const int begin = blockIdx.x * a.stretch, end = min(a.rows, begin + a.stretch);
    for (int from = begin; from < end;) {
        const At start = at_row(from, a);
        const int to = a.gate ? min(end, from + (int)a.pixels - start.pixel) : end;
        const float* gate = a.gate ? a.gate + (int64_t)start.sample * a.C : nullptr;
        // what dh is multiplied with on its way to the normalised block
        Eight k = parameter<V>(a.post_weight, 1.0f, lane, a);
        const Eight sc = parameter<V>(a.scale, 1.0f, lane, a), ga = parameter<V>(gate, 1.0f, lane, a);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) k.v[i] = mul(k.v[i], mul(sc.v[i], ga.v[i]));

        for (int k = 0; k < R - 1; ++k) ask(from + k * here, to, k);
        int slot = 0;
        for (int base = from; base < to; base += here) {
            const int row = base + mine;
            const bool there = row < to;
            const At at = at_row(there ? row : base, a);
            ask(base + (R - 1) * here, to, slot == 0 ? R - 1 : slot - 1);
            copies_wait<R - 1>();
            const char* place = ring + slot * round;
            slot = slot == R - 1 ? 0 : slot + 1;
            const TX* h_row = row_of<TX>(a.x, at, a.x_pixel, a.x_sample);
            Eight h = zero, b = zero;
            if (pre) h = widened(X::get(place + h_at, h_row, lane, a, there));
            if (a.b) b = widened(B::get(place + b_at, row_of<TB>(a.b, at, a.b_pixel, a.b_sample), lane, a, there));
            // both norms
            float2 mean = make_float2(0.0f, 0.0f);
            if (a.pre == PP_NORM_LAYER || a.post == PP_NORM_LAYER) {
                mean = sum(make_float2(a.pre == PP_NORM_LAYER ? across(sum_of(h)) : 0.0f, a.post == PP_NORM_LAYER ? across(sum_of(b)) : 0.0f));
                mean = mul(mean, both(a.inv_c));
            }
            if (a.pre == PP_NORM_LAYER) centre<V>(h, mean.x, lane, a);
            if (a.post == PP_NORM_LAYER) centre<V>(b, mean.y, lane, a);
            float2 both_sums[2] = {make_float2(across(sum_of(h)), across(sum_of(b))), make_float2(dot(h, h), dot(b, b))};
            if (pre || post) sum.all(both_sums);
            const Scaling sh(a.pre, both_sums[0].x, both_sums[1].x, a), sb(a.post, both_sums[0].y, both_sums[1].y, a);
            const float2 r = there ? make_float2(sh.root, sb.root) : make_float2(0.0f, 0.0f);
            const float2 shift = there ? make_float2(sh.shift, sb.shift) : make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < E / 2; ++i)
                h.v[i] = fma(h.v[i], both(r.x), both(shift.x)), b.v[i] = fma(b.v[i], both(r.y), both(shift.y));
            Eight d = zero;
            if (!pre && a.dh) d = widened(X::get(place + d_at, row_of<TX>(a.dh, at, a.dh_pixel, a.dh_sample), lane, a, there));
            if (pre) {
                Eight dz = widened(B::get(place + y_at, row_of<TB>(a.dy, at, a.dy_pixel, a.dy_sample), lane, a, there));
                if (a.act == PP_ACT_RELU) {
                    // fp32's z is off by less than 2^-18 of its terms' sizes (each value, the mean, and the root by some 16 roundings
                    // of the row's sums): there the sign is taken in 64 bits
                    bool close = false;
                    unsigned above = 0;
                    const float* hf = reinterpret_cast<const float*>(h.v);
                    const float* wf = reinterpret_cast<const float*>(w.v);
                    const float* bf = reinterpret_cast<const float*>(bias.v);
                    const float spread = 1.0f + 2.0f * fabsf(mean.x) * r.x;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float z = fmaf(hf[e], wf[e], bf[e]);
                        above |= (unsigned)(z > 0.0f) << e;
                        close |= fabsf(z) <= 3.8147e-6f * (fabsf(wf[e]) * (fabsf(hf[e]) + spread) + fabsf(bf[e])) && inside<V>(lane, a, e);
                    }
                    close = close && there;
                    if (WIDE ? __syncthreads_or(close) : __any_sync(0xffffffffu, close)) 
                        above = above_zero<TX, V, WIDE>(place + h_at, h_row, there, a, lane, sum);
                    float* f = reinterpret_cast<float*>(dz.v);
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (!(above >> e & 1)) f[e] = 0.0f;
                } else if (a.act == PP_ACT_SILU) {
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
                float2 q = sum(make_float2(a.pre == PP_NORM_LAYER ? across(sum_of(t)) : 0.0f, dot(t, h)));
                q = mul(q, both(a.inv_c));
                if (a.dh) d = widened(X::get(place + d_at, row_of<TX>(a.dh, at, a.dh_pixel, a.dh_sample), lane, a, there));
#pragma unroll
                for (int i = 0; i < E / 2; ++i)
                    d.v[i] = fma(fma(h.v[i], both(-q.y), add(t.v[i], both(-q.x))), both(r.x), d.v[i]);
            }
            if (a.dx) put(dense_row<TX>(a.dx, row, a), narrowed<TX, V>(d), lane, a, there);
            if (!a.b) continue;
            Eight t;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                const float2 live = there ? d.v[i] : make_float2(0.0f, 0.0f);
                s_e.v[i] = fma(live, b.v[i], s_e.v[i]);
                s_f.v[i] = add(live, s_f.v[i]);
                t.v[i] = mul(d.v[i], k.v[i]);
            }
            if (post) {
                float2 q = sum(make_float2(a.post == PP_NORM_LAYER ? across(sum_of(t)) : 0.0f, dot(t, b)));
                q = mul(q, both(a.inv_c));
#pragma unroll
                for (int i = 0; i < E / 2; ++i) t.v[i] = mul(fma(b.v[i], both(-q.y), add(t.v[i], both(-q.x))), both(r.y));
            }
            put(dense_row<TB>(a.db, row, a), narrowed<TB, V>(t), lane, a, there);
        }

        // the sample's sums: of the block's norm, the gate and the scale
        if (a.b) {
            float* e_all = lanes_sum;
            float* f_all = lanes_sum + kBlockThreads * E;
            if (!WIDE) {
                __syncthreads();
                const float* pe = reinterpret_cast<const float*>(s_e.v);
                const float* pf = reinterpret_cast<const float*>(s_f.v);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int c = channel<V>(lane, a.threads, i);
                    e_all[mine * a.threads * E + c] = pe[i];
                    f_all[mine * a.threads * E + c] = pf[i];
                }
                __syncthreads();
            }
            const bool first = from == begin, whole = (first ? start.pixel == 0 : true) && (to < end || at_row(end - 1, a).pixel == a.pixels - 1);
#pragma unroll
            for (int i = 0; i < OWN; ++i) {
                const int c = WIDE ? channel<V>(lane, a.threads, i) : threadIdx.x;
                if (c >= a.C) continue;
                float e = 0, f = 0;
                if (WIDE) {
                    e = reinterpret_cast<const float*>(s_e.v)[i];
                    f = reinterpret_cast<const float*>(s_f.v)[i];
                } else {
                    for (int g = 0; g < here; ++g) e += e_all[g * a.threads * E + c], f += f_all[g * a.threads * E + c];
                }
                const float ga_c = gate ? gate[c] : 1.0f, sc_c = a.scale ? a.scale[c] : 1.0f;
                const float joined = fmaf(a.post_weight ? a.post_weight[c] : 1.0f, e, a.post_bias ? a.post_bias[c] * f : 0.0f);
                total(0, i) = fmaf(sc_c * ga_c, e, total(0, i));
                total(1, i) = fmaf(sc_c * ga_c, f, total(1, i));
                total(2, i) = fmaf(ga_c, joined, total(2, i));
                if (a.dgate) {
                    if (whole)
                        a.dgate[(int64_t)start.sample * a.C + c] = sc_c * joined;
                    else
                        a.gates[((int64_t)blockIdx.x * 2 + !first) * a.C + c] = sc_c * joined;
                }
            }
            s_e = s_f = zero;
        }
        from = to;
    }

    // the CTA's sums
    float* out = a.sums + (int64_t)blockIdx.x * kBlockSums * a.C;
    if (!WIDE) {
        __syncthreads();
        const float* pw = reinterpret_cast<const float*>(s_w.v);
        const float* pb = reinterpret_cast<const float*>(s_b.v);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int c = channel<V>(lane, a.threads, i);
            lanes_sum[mine * a.threads * E + c] = pw[i];
            lanes_sum[kBlockThreads * E + mine * a.threads * E + c] = pb[i];
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int c = WIDE ? channel<V>(lane, a.threads, i) : threadIdx.x;
        if (c >= a.C) continue;
        float e = 0, f = 0;
        if (WIDE) {
            e = reinterpret_cast<const float*>(s_w.v)[i];
            f = reinterpret_cast<const float*>(s_b.v)[i];
        } else {
            for (int g = 0; g < here; ++g) e += lanes_sum[g * a.threads * E + c], f += lanes_sum[kBlockThreads * E + g * a.threads * E + c];
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
template <typename TX, typename TB, int V, bool WIDE>
cudaError_t forward_rows(const BlockArgs& a, int threads, int ctas, cudaStream_t st) {
    constexpr int kRound = Ahead<TX, V>::kBytes + Ahead<TB, V>::kBytes;
    static std::atomic<uint64_t> allowed{0};
    if (const cudaError_t e = allow_shared(block_rows<TX, TB, V, WIDE>, allowed, kRounds * kRound * (WIDE ? 512 : kBlockThreads))) return e;
    block_rows<TX, TB, V, WIDE><<<ctas, threads, kRounds * kRound * threads, st>>>(a);
    return cudaGetLastError();
}
template <typename TX, typename TB, int V>
cudaError_t forward_as(const BlockArgs& a, cudaStream_t st) {
    if (a.threads > 32) return forward_rows<TX, TB, V, true>(a, a.threads, std::min(a.rows, 152 * std::max(1, 768 / a.threads)), st);
    const int here = kBlockThreads / a.threads;
    return forward_rows<TX, TB, V, false>(a, kBlockThreads, std::min((a.rows + here - 1) / here, 152 * 3), st);
}
template <typename TX, typename TB, int V, bool WIDE>
cudaError_t backward_rows(const BlockArgs& a, int threads, cudaStream_t st) {
    constexpr int kEach = kRoundsBack<TX, TB, WIDE> * 2 * (Ahead<TX, V>::kBytes + Ahead<TB, V>::kBytes) + 3 * (WIDE ? E : 1) * (int)sizeof(float);   // of a thread
    static std::atomic<uint64_t> allowed{0};
    if (const cudaError_t e = allow_shared(block_back_rows<TX, TB, V, WIDE>, allowed, kEach * (WIDE ? 512 : kBlockThreads))) return e;
    block_back_rows<TX, TB, V, WIDE><<<a.ctas, threads, kEach * threads, st>>>(a);
    return cudaGetLastError();
}
template <typename TX, typename TB, int V>
cudaError_t backward_as(const BlockArgs& a, cudaStream_t st) {
    if (const cudaError_t e = a.threads > 32 ? backward_rows<TX, TB, V, true>(a, a.threads, st) : backward_rows<TX, TB, V, false>(a, kBlockThreads, st))
        return e;
    return block_join(a, st);
}

}  // namespace

template <typename TX, typename TB>
cudaError_t BlockKernels<TX, TB>::forward(const BlockArgs& a, int V, cudaStream_t st) {
    return V == 8 ? forward_as<TX, TB, 8>(a, st) : V == 2 ? forward_as<TX, TB, 2>(a, st) : forward_as<TX, TB, 1>(a, st);
}
template <typename TX, typename TB>
cudaError_t BlockKernels<TX, TB>::backward(const BlockArgs& a, int V, cudaStream_t st) {
    return V == 8 ? backward_as<TX, TB, 8>(a, st) : V == 2 ? backward_as<TX, TB, 2>(a, st) : backward_as<TX, TB, 1>(a, st);
}

}  // namespace patconv
