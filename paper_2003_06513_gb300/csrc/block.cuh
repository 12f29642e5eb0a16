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
__device__ __forceinline__ Vec<T, V> load_wide(const T* p) {
    if constexpr (sizeof(T) * V > 16) {               // eight fp32 values: two vectors
        Vec<T, V> r;
        const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
        memcpy(&r, &a, 16);
        memcpy(&r.v[4], &b, 16);
        return r;
    } else {
        return load<T, V>(p);
    }
}
template <typename T, int V>
struct Raw {                                          // as it is read
    Vec<T, V> v[E / V];
};
template <typename T, int V>
__device__ __forceinline__ void fetch(Raw<T, V>& r, const T* row, int lane, const BlockArgs& a, bool there) {
#pragma unroll
    for (int j = 0; j < E / V; ++j) {
        const int at = lane + j * a.threads;
        if (there && at < a.vectors)
            r.v[j] = load_wide<T, V>(row + (int64_t)at * V);
        else
            r.v[j] = Vec<T, V>{};
    }
}
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
__global__ void __launch_bounds__(WIDE ? 512 : kBlockThreads) block_rows(BlockArgs a) {
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

    for (int base = blockIdx.x * here; base < a.rows; base += gridDim.x * here) {
        const int row = base + mine;
        const bool there = row < a.rows;
        const At at = at_row(there ? row : 0, a);
        Raw<TX, V> rx;
        Raw<TB, V> rb;
        if (a.x) fetch(rx, row_of<TX>(a.x, at, a.x_pixel, a.x_sample), lane, a, there);
        if (a.b) fetch(rb, row_of<TB>(a.b, at, a.b_pixel, a.b_sample), lane, a, there);
        if (a.gate && there && at.sample != gate_of) {
            gate = parameter<V>(a.gate + (int64_t)at.sample * a.C, 1.0f, lane, a);
            gate_of = at.sample;
        }
        Eight h = widened(rx);
        if (a.b) {
            Eight b = widened(rb);
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
template <int V, bool WIDE>
__device__ __noinline__ unsigned above_zero(Eight h, const BlockArgs& a, int lane, RowSum<WIDE>& sum) {
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
    __shared__ float2 scratch[WIDE ? 64 : 1];
    __shared__ float lanes_sum[WIDE ? 1 : 2 * kBlockThreads * E];
    const int lane = WIDE ? threadIdx.x : threadIdx.x % a.threads;
    const int here = WIDE ? 1 : kBlockThreads / a.threads, mine = WIDE ? 0 : threadIdx.x / a.threads;
    RowSum<WIDE> sum{a.threads, scratch};
    const bool pre = a.pre != PP_NORM_NONE, post = a.post != PP_NORM_NONE;
    const Eight w = parameter<V>(a.weight, 1.0f, lane, a), bias = parameter<V>(a.bias, 0.0f, lane, a);
    const Eight zero{};
    Eight s_w = zero, s_b = zero, s_e = zero, s_f = zero;        // sums of dz h^, dz, and of a sample dh b^, dh
    // the sums over all samples that the threads of channel c hold (not WIDE: thread c; WIDE: the thread's eight)
    constexpr int OWN = WIDE ? E : 1;
    float t_pw[OWN] = {}, t_pb[OWN] = {}, t_s[OWN] = {};

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

        for (int base = from; base < to; base += here) {
            const int row = base + mine;
            const bool there = row < to;
            const At at = at_row(there ? row : from, a);
            Raw<TX, V> rd, rh;
            Raw<TB, V> ry, rb;
            if (a.dh) fetch(rd, row_of<TX>(a.dh, at, a.dh_pixel, a.dh_sample), lane, a, there);
            if (a.b) fetch(rb, row_of<TB>(a.b, at, a.b_pixel, a.b_sample), lane, a, there);
            if (pre) {
                fetch(rh, row_of<TX>(a.x, at, a.x_pixel, a.x_sample), lane, a, there);
                fetch(ry, row_of<TB>(a.dy, at, a.dy_pixel, a.dy_sample), lane, a, there);
            }
            Eight d = a.dh ? widened(rd) : zero, b = a.b ? widened(rb) : zero, h = pre ? widened(rh) : zero;
            // both norms
            float2 mean = make_float2(0.0f, 0.0f);
            if (a.pre == PP_NORM_LAYER || a.post == PP_NORM_LAYER) {
                mean = sum(make_float2(a.pre == PP_NORM_LAYER ? across(sum_of(h)) : 0.0f, a.post == PP_NORM_LAYER ? across(sum_of(b)) : 0.0f));
                mean = mul(mean, both(a.inv_c));
            }
            const Eight h0 = h;
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
            if (pre) {
                Eight dz = widened(ry);
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
                    if (WIDE ? __syncthreads_or(close) : __any_sync(0xffffffffu, close)) above = above_zero<V, WIDE>(h0, a, lane, sum);
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
                t_pw[i] = fmaf(sc_c * ga_c, e, t_pw[i]);
                t_pb[i] = fmaf(sc_c * ga_c, f, t_pb[i]);
                t_s[i] = fmaf(ga_c, joined, t_s[i]);
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
        out[2 * a.C + c] = t_pw[i];
        out[3 * a.C + c] = t_pb[i];
        out[4 * a.C + c] = t_s[i];
    }
}

template <typename TX, typename TB, int V>
cudaError_t forward_as(const BlockArgs& a, cudaStream_t st) {
    if (a.threads > 32) {
        const int ctas = std::min(a.rows, 152 * std::max(1, 1536 / a.threads));
        block_rows<TX, TB, V, true><<<ctas, a.threads, 0, st>>>(a);
    } else {
        const int here = kBlockThreads / a.threads, ctas = std::min((a.rows + here - 1) / here, 152 * 4);
        block_rows<TX, TB, V, false><<<ctas, kBlockThreads, 0, st>>>(a);
    }
    return cudaGetLastError();
}
template <typename TX, typename TB, int V>
cudaError_t backward_as(const BlockArgs& a, cudaStream_t st) {
    if (a.threads > 32)
        block_back_rows<TX, TB, V, true><<<a.ctas, a.threads, 0, st>>>(a);
    else
        block_back_rows<TX, TB, V, false><<<a.ctas, kBlockThreads, 0, st>>>(a);
    if (const cudaError_t e = cudaGetLastError()) return e;
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
